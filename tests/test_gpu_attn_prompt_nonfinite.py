"""Values that are not finite in prompts: with finite keys they reach exactly their own dim of exactly the rows that see
them, as what a sum with positive weights makes of them, and leave every other bit as it is."""
import numpy as np
import pytest

from test_gpu_attn_prompt import DEV, DT, cum, ints, make, u  # noqa: F401  (u is a fixture)

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
INF, NAN = float("inf"), float("nan")


def run(u, q, k, v, nq, nk, causal):
    return u.attn_prompt(q.to(DEV), k.to(DEV), v.to(DEV), ints(cum(nq)), ints(cum(nk)), causal=causal).cpu()


def check(u, q, k, v, nq, nk, places, causal=True):
    """places: (sequence, token, key head, dim, value)."""
    HQ, H = q.shape[1], k.shape[1]
    cq, ck = cum(nq), cum(nk)
    clean = run(u, q, k, v, nq, nk, causal)
    up = np.zeros(clean.shape, dtype=bool)
    down = up.copy()
    bad = v.clone()
    for (b, token, head, dim), value in {p[:4]: p[4] for p in places}.items():  # (of two at one place the last one)
        bad[ck[b] + token, head, dim] = value
        first = max(0, token - (nk[b] - nq[b])) if causal else 0  # of the rows that see it
        rows, heads = slice(cq[b] + first, cq[b + 1]), slice(head * HQ // H, (head + 1) * HQ // H)
        up[rows, heads, dim] |= not value == -INF
        down[rows, heads, dim] |= not value == INF
    got = run(u, q, k, bad, nq, nk, causal).float().numpy()
    assert np.array_equal(np.isnan(got), up & down)
    assert np.array_equal(got == INF, up & ~down) and np.array_equal(got == -INF, down & ~up)
    fine = ~(up | down)
    assert fine.any() and np.array_equal(got[fine], clean.float().numpy()[fine])


def some_places(rng, nk, H, D, count):
    """Random ones, both signs in one dim among them, and all kinds of them in the last tile."""
    p = []
    for _ in range(count):
        b = int(rng.integers(len(nk)))
        if nk[b]:
            p.append((b, int(rng.integers(nk[b])), int(rng.integers(H)), int(rng.integers(D)), [INF, -INF, NAN][rng.integers(3)]))
    b = int(np.argmax(nk))
    n = nk[b]
    for i, value in enumerate((INF, -INF, NAN)):
        p.append((b, n - 1 - i, 0, (7 * i + 3) % D, value))
    p += [(b, n - 1, 0, D - 1, INF), (b, max(0, n - 5), 0, D - 1, -INF)]
    return p


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("HQ,H", [(1, 1), (6, 2), (5, 1)])
@pytest.mark.parametrize("nq,nk", [([200], [200]), ([64], [64]), ([40, 0, 129], [100, 3, 150]), ([1, 77], [70, 77])])
def test_random_places(u, dtype, D, HQ, H, nq, nk):  # noqa: F811
    q, k, v = make(nq, nk, HQ, H, D, dtype, seed=D + HQ, std=1.0)
    rng = np.random.default_rng(D + HQ + nq[0])
    for count in (0, 4, 30):
        check(u, q, k, v, nq, nk, some_places(rng, nk, H, D, count))


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("D", [64, 128])
def test_every_dim_and_row_of_a_tile(u, dtype, D):  # noqa: F811
    """One value at a time, over the dims at one token and over the tokens at one dim of the tile that is partly seen."""
    nq = [64]
    q, k, v = make(nq, nq, 2, 1, D, dtype, seed=D, std=1.0)
    for dim in range(D):
        check(u, q, k, v, nq, nq, [(0, 37, 0, dim, (INF, -INF, NAN)[dim % 3])])
    for token in range(64):
        check(u, q, k, v, nq, nq, [(0, token, 0, 5, (INF, -INF, NAN)[token % 3])])


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("D", [64, 128])
def test_parts_of_keys(u, causal, D):  # noqa: F811
    """Few queries before many keys: the parts are joined."""
    nq, nk = [6, 70], [1500, 2000]
    assert u.attn_prompt_workspace_bytes(2, 76, 3500, 4, 1, D) > 0
    q, k, v = make(nq, nk, 4, 1, D, "bf16", seed=D, std=1.0)
    rng = np.random.default_rng(D)
    for count in (0, 12):
        check(u, q, k, v, nq, nk, some_places(rng, nk, 1, D, count), causal)


def test_where_all_is_seen(u):  # noqa: F811
    nq, nk = [100, 3], [90, 200]
    q, k, v = make(nq, nk, 4, 2, 128, "f16", seed=3, std=1.0)
    check(u, q, k, v, nq, nk, some_places(np.random.default_rng(3), nk, 2, 128, 10), causal=False)
