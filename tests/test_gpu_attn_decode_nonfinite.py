"""Values that are not finite in 16-bit pages: with finite keys they reach exactly their own dim of exactly the new tokens
that see them, as what a sum with positive weights makes of them, and leave every other bit as it is.  In code caches a
scale that is not a number takes its head (8 bits) or its half of it (4 bits) along."""
import numpy as np
import pytest

from test_gpu_attn_decode import DEV, DT, filled, ints, u  # noqa: F401  (u is a fixture)

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
INF, NAN = float("inf"), float("nan")
PAGE = 16


@pytest.mark.parametrize("kind", ["f16", "bf16"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("H,group,q_len", [(1, 1, 4), (2, 3, 2), (1, 8, 7), (2, 1, 16)])
@pytest.mark.parametrize("n", [20, 70, 300, 2000])
def test_values_in_their_place(u, kind, D, H, group, q_len, n):  # noqa: F811
    cache, pt, _ = filled(u, kind, [n], PAGE, H, D, seed=n + D, spread=0.0)
    q = torch.randn((1, q_len, H * group, D), generator=torch.Generator().manual_seed(1)).to(DT[kind]).to(DEV)
    lens = ints([n])
    clean = u.attn_decode(q, cache, pt, lens)[0].cpu()
    rng = np.random.default_rng(n + D + q_len)
    for count in (1, 8, 60):
        v = cache[1].clone()
        place = {}
        for i in range(count):
            token = n - 1 - int(rng.integers(min(n, q_len + 3))) if i % 3 else int(rng.integers(n))
            place[token, int(rng.integers(H)), int(rng.integers(D))] = (INF, -INF, NAN)[rng.integers(3)]
        up = np.zeros(clean.shape, dtype=bool)
        down = up.copy()
        for (token, head, dim), value in place.items():
            v[int(pt[0, token // PAGE]), head, token % PAGE, dim] = value
            rows, heads = slice(max(0, token - (n - q_len)), None), slice(head * group, (head + 1) * group)
            up[rows, heads, dim] |= not value == -INF
            down[rows, heads, dim] |= not value == INF
        got = u.attn_decode(q, (cache[0], v, None, None), pt, lens)[0].cpu().float().numpy()
        assert np.array_equal(np.isnan(got), up & down)
        assert np.array_equal(got == INF, up & ~down) and np.array_equal(got == -INF, down & ~up)
        fine = ~(up | down)
        assert np.array_equal(got[fine], clean.float().numpy()[fine])


@pytest.mark.parametrize("kind", ["i8", "i4"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("n", [20, 300, 2000])
def test_scales_in_their_place(u, kind, D, n):  # noqa: F811
    H, group, q_len = 2, 3, 4
    cache, pt, _ = filled(u, kind, [n], PAGE, H, D, seed=n + D, spread=0.0)
    q = torch.randn((1, q_len, H * group, D), generator=torch.Generator().manual_seed(2)).bfloat16().to(DEV)
    lens = ints([n])
    clean = u.attn_decode(q, cache, pt, lens)[0].cpu()
    for token in (n - 1, n - 2, n - 4, n - 5, 3):
        for head in range(H):
            for half in range(2 if kind == "i4" else 1):
                scales = cache[3].clone()
                at = (int(pt[0, token // PAGE]), head, token % PAGE)
                scales[at if kind == "i8" else (*at, half)] = NAN
                got = u.attn_decode(q, (*cache[:3], scales), pt, lens)[0].cpu()
                bad = torch.zeros(clean.shape, dtype=torch.bool)
                dims = slice(None) if kind == "i8" else slice(half * D // 2, (half + 1) * D // 2)
                first = max(0, token - (n - q_len))
                bad[first:, head * group:(head + 1) * group, dims] = True
                assert torch.equal(torch.isnan(got), bad)
                assert torch.equal(got[:first], clean[:first])
                # the other half's unit may be another one: operands below 2^-14 of it lose other bits
                assert torch.allclose(got[~bad].float(), clean[~bad].float(), rtol=2.0 ** -7, atol=2.0 ** -12)
