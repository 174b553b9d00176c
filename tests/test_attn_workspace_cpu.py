"""Workspace sizes of attention over the cache, against what its calls ask for."""
import itertools
import os

import pytest

import paper_2606_10520_amd.unisvq as u

pytestmark = pytest.mark.skipif(not os.path.exists(u.LIB_PATH), reason="libunisvq.so not built")

EWORKSPACE = -6
GOOD = 0x10000
LENS = [1, 100, 128, 129, 1000, 1024, 1025, 1100, 2000, 8192, 40000, 1 << 20, 1 << 30]


def size(sequences, q_len, q_heads, kv_heads, head_dim, max_len):
    return u.load().unisvq_attn_decode_workspace_bytes(sequences, q_len, q_heads, kv_heads, head_dim, max_len)


def asks_for_workspace(sequences, q_len, q_heads, kv_heads, head_dim, max_len, width, kind=u.CACHE_F16):
    """Whether a call without a workspace is refused for that (so nothing is launched)."""
    c = u.Cache(8, 16, kv_heads, head_dim, kind, GOOD, GOOD, GOOD, GOOD)
    return u.load().unisvq_attn_decode(c, GOOD, sequences, width, GOOD, max_len, q_len, q_heads, GOOD, q_heads * head_dim,
                                       head_dim, u.F16, 0.1, GOOD, q_heads * head_dim, head_dim, None, None, 0,
                                       None) == EWORKSPACE


SHAPES = list(itertools.product([1, 3, 16, 300], [1, 5], [(8, 8), (64, 8), (32, 32), (150, 150)], [64, 128]))


@pytest.mark.parametrize("sequences,q_len,heads,head_dim", SHAPES)
def test_a_larger_max_len_never_needs_less(sequences, q_len, heads, head_dim):
    sizes = [size(sequences, q_len, *heads, head_dim, n) for n in LENS]
    assert sizes == sorted(sizes)


@pytest.mark.parametrize("sequences,q_len,heads,head_dim", SHAPES)
def test_the_size_without_a_max_len_serves_every_width(sequences, q_len, heads, head_dim):
    """max_len 0 is the page table's whole width, which the size function does not know."""
    assert size(sequences, q_len, *heads, head_dim, 0) == max(size(sequences, q_len, *heads, head_dim, n) for n in LENS) > 0


def test_calls_ask_for_the_size_of_the_width():
    for width in (65, 100, 600):
        need = size(1, 1, 8, 8, 128, 16 * width)
        assert need > 0 and asks_for_workspace(1, 1, 8, 8, 128, 0, width)
        assert need <= size(1, 1, 8, 8, 128, 0)


@pytest.mark.parametrize("q_len,heads,slots", [(16, (65535, 65535), 3), (16, (65535, 1), 3), (1, (8, 8), 66), (1, (1024, 1024), 3)])
def test_the_largest_counts_do_not_overflow(q_len, heads, slots):
    """fp32 sums, a maximum and a sum for each part of each row, and the words that say where sequences begin."""
    n = 2 ** 31 - 1
    assert size(n, q_len, *heads, 128, 1 << 30) == n * q_len * heads[0] * slots * 130 * 4 + (n + 2) * 4
