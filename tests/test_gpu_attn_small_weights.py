"""Many keys of small weight: what f16 weights lose of them."""
import numpy as np
import pytest

from test_gpu_attn_decode_ranges import along, coded
from test_gpu_attn_prompt import DEV, DT, ints, u  # noqa: F401  (u is a fixture)

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("op", ["prompt", "pages", "i8", "i4"])
@pytest.mark.parametrize("down", [22, 26, 28])
def test_one_key_of_no_value_and_many_of_small_weight(u, op, dtype, D, down):  # noqa: F811
    """The first key's weight is 1 and its value 0, the others' weights are about 2^-down and their values about 1."""
    n, page = 60001, 256
    rng = np.random.default_rng(down)
    s = -np.log(2) * (down + rng.uniform(-0.5, 0.5, n))
    s[0] = 0
    v = rng.uniform(0.5, 1, (n, 1, D))
    v[0] = 0
    k = along(s, 1, D)
    q = torch.zeros((1, 2, D))
    q[:, :, 0] = 1
    q = q.to(DT[dtype])
    if op in ("i8", "i4"):
        cache, pt, (k, v) = coded(op, k, v, page)
        out = u.attn_decode(q.to(DEV), cache, pt, ints([n]), scale=1.0)
    else:
        k, v = torch.from_numpy(k).to(DT[dtype]), torch.from_numpy(v).to(DT[dtype])
        if op == "prompt":
            out = u.attn_prompt(q.to(DEV), k.to(DEV), v.to(DEV), ints([0, 1]), ints([0, n]), causal=False, scale=1.0)
        else:
            pages = -(-n // page)
            pools = [torch.ones((pages * page, 1, D), dtype=DT[dtype]) for _ in range(2)]
            for pool, x in zip(pools, (k, v)):
                pool[:n] = x
            cache = (*[p.view(pages, page, 1, D).transpose(1, 2).contiguous().to(DEV) for p in pools], None, None)
            out = u.attn_decode(q.to(DEV), cache, ints(np.arange(pages)[None]), ints([n]), scale=1.0)
        k, v = k.double().numpy(), v.double().numpy()
    p = np.exp(k[:, 0, 0])
    want = (p[:, None] * v[:, 0]).sum(0) / p.sum()
    # a weight's rounding: 2^-9 (bf16) or 2^-12, or half of f16's smallest step in a unit where the largest is 2^7 or
    # more, 2^-32; scores to 2^-19 of up to 20; the fp32 sums by n 2^-24 of them at most; the result to 16 bits once
    bound = want * (2.0 ** -8 + 2.0 ** -16 + n * 2.0 ** -24) + n * 2.0 ** -32
    assert np.all(np.abs(out[0].double().cpu().numpy() - want) <= bound)
