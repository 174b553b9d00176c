"""The kernels of 4-bit products that the library holds: those that some call takes, and no others."""
import os
import re

import pytest

import paper_2606_10520_amd.unisvq as u

built = pytest.mark.skipif(not os.path.exists(u.LIB_PATH), reason="libunisvq.so not built")


@built
def test_variants_of_few_tokens():
    """Kernels of (tokens, wavefronts, tiles asked for together): eight tokens are taken with 16 to 32 groups of columns alone."""
    with open(u.LIB_PATH, "rb") as f:
        names = set(re.findall(rb"few_kernelI(DF16_|DF16b|u6__bf16|a)Li(\d+)ELi(\d+)ELi(\d+)E", f.read()))
    have = {tuple(map(int, n[1:])) for n in names}
    want = {(t, 8, d) for t in (1, 2, 4) for d in range(1, 6)} | {(t, 16, d) for t in (1, 2, 4) for d in (2, 3, 4)}
    assert have == want | {(8, 8, 2), (8, 8, 3), (8, 8, 4), (8, 16, 2)}
    assert len(names) == 3 * len(want) + 2 * 4
