"""Attention over 8- and 4-bit caches whose values' scales lie far apart: a result is bound by the tokens that its row
sees, by their weights times their values, and by its own half of the head."""
import numpy as np
import pytest

import attn_ref as ref

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.fixture(scope="module")
def u():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2606_10520_amd.unisvq as u
    u.load()
    return u


def ints(v):
    return torch.tensor(np.asarray(v), dtype=torch.int32, device=DEV)


def coded(kind, k, v, page=32):
    """One sequence's k and v [len][H][D] as a cache, its page table, and the values held, fp64."""
    n, H, D = k.shape
    pages = -(-n // page)
    pools, scales, held = [], [], []
    for x in (k, v):
        x = np.concatenate([x, np.ones((pages * page - n, H, D))]).astype(np.float32)
        code, scale = ref.quantise(x, kind)
        held.append(ref.dequantise(code, scale, kind).astype(np.float64)[:n])
        code, scale = (np.swapaxes(y.reshape(pages, page, *y.shape[1:]), 1, 2) for y in (code, scale))
        if kind == "i4":
            c = (code + 8).astype(np.uint8)
            code = c[..., 0::2] | c[..., 1::2] << 4
        pools.append(torch.from_numpy(np.ascontiguousarray(code)).to(DEV))
        s = torch.from_numpy(np.ascontiguousarray(scale))
        scales.append((s.bfloat16() if kind == "i4" else s).to(DEV))
    return (*pools, *scales), ints(np.arange(pages)[None]), held


def attend_and_check(u, kind, q, k, v, scale, rows=None, spoil=()):
    """q [q_len][HQ][D] bf16.  Every row is checked against 64 bits on the tokens that it sees.  `rows`: those to check;
    spoil: tokens whose value scales are made NaN.  What a weight's rounding to f16 loses absolutely (2^-25 of a unit
    that the largest product of a weight and a token's largest value sets, a factor of 4 for that value's place in the
    unit) is counted for the row's own products, and for a half of the head by itself in a 4-bit cache."""
    cache, pt, (hk, hv) = coded(kind, k, v)
    n, (q_len, HQ, D), H = k.shape[0], q.shape, k.shape[1]
    for t in spoil:
        cache[3][t // 32, :, t % 32] = float("nan")
    lse = torch.empty((1, q_len, HQ), device=DEV)
    out = u.attn_decode(q[None].to(DEV), cache, pt, ints([n]), scale=scale, lse=lse)[0]
    for j in range(q_len) if rows is None else rows:
        seen = n - q_len + 1 + j
        qj, kj, vj = q[j:j + 1].double().numpy(), hk[:seen], hv[:seen]
        r = ref.attention(qj, kj, vj, [seen - 1], scale)
        parts = 2 if kind == "i4" else 1
        halves = np.abs(vj).reshape(seen, H, parts, D // parts).max(-1)  # [token][head][half]
        most = np.zeros((1, HQ, D))
        for h in range(HQ):
            s = scale * (kj[:, h * H // HQ] @ qj[0, h])
            p = np.exp(s - r[1][0, h])
            most[0, h] = np.repeat((p[:, None] * halves[:, h * H // HQ]).max(0, initial=0), D // parts)
        ref.check(out[j:j + 1].double().cpu().numpy(), lse[0, j:j + 1].double().cpu().numpy(), r, seen, "f16", "bf16", most)
    return out


def along(values, H, D):
    """Keys whose first dim is `values` [len] and all others zero."""
    k = np.zeros((len(values), H, D), dtype=np.float32)
    k[:, :, 0] = np.asarray(values)[:, None]
    return k


KINDS = ["i8", "i4"]


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("n", [6, 37, 300, 1500])
@pytest.mark.parametrize("up", [20, 25, 30, 60, -40])
def test_larger_values_of_tokens_not_seen(u, kind, n, up):
    rng = np.random.default_rng(n)
    k, v = rng.standard_normal((2, n, 2, 128))
    v[n - 1] *= 2.0 ** up
    v[n - 2] *= 2.0 ** (up / 2)
    q = torch.from_numpy(rng.standard_normal((4, 6, 128))).bfloat16()
    attend_and_check(u, kind, q, k, v, 0.1)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("n", [5, 20, 260])
@pytest.mark.parametrize("up", [-60, -20, 0, 20, 60])
def test_scales_that_are_not_finite_where_not_seen(u, kind, n, up):
    rng = np.random.default_rng(n)
    k, v = rng.standard_normal((2, n, 1, 64))
    q = torch.from_numpy(rng.standard_normal((3, 4, 64))).bfloat16()
    out = attend_and_check(u, kind, q, k, v * 2.0 ** up, 0.1, rows=[0, 1], spoil=[n - 1])
    assert torch.isnan(out[2]).all()


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("at", [0, 50, 199])
@pytest.mark.parametrize("up,down", [(26, 40), (40, 60), (20, 10), (100, 110)])
def test_large_values_of_small_weight(u, kind, at, up, down):
    """A value 2^up larger whose weight is 2^-down of the others': the others are what counts, or share in it."""
    rng = np.random.default_rng(at)
    v = rng.standard_normal((200, 2, 128))
    v[at] *= 2.0 ** up
    s = np.zeros(200)
    s[at] = -down * np.log(2)
    q = torch.zeros((1, 2, 128))
    q[:, :, 0] = 1
    attend_and_check(u, kind, q.bfloat16(), along(s, 2, 128), v, 1.0)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("step", [0.9, -0.9, 3.0, -3.0])
def test_scores_and_values_that_cancel(u, kind, step):
    """Weights rise (or fall) by 2^step a token and values fall (or rise) as much: all tokens count alike."""
    n = int(90 / abs(step))
    rng = np.random.default_rng(1)
    t = np.arange(n) - n // 2
    v = rng.standard_normal((n, 1, 128)) * 2.0 ** (-step * t)[:, None, None]
    q = torch.zeros((2, 1, 128))
    q[:, :, 0] = 1
    attend_and_check(u, kind, q.bfloat16(), along(t * step * np.log(2), 1, 128), v, 1.0)


@pytest.mark.parametrize("kind", KINDS)
def test_zeros_of_large_weight(u, kind):
    """The token that takes all weight but 2^-60 has values of zero."""
    rng = np.random.default_rng(2)
    v = rng.standard_normal((70, 1, 64))
    s = np.zeros(70)
    for at in (0, 33, 69):
        w, z = v.copy(), s.copy()
        w[at], z[at] = 0, 60 * np.log(2)
        q = torch.zeros((1, 1, 64))
        q[:, :, 0] = 1
        attend_and_check(u, kind, q.bfloat16(), along(z, 1, 64), w, 1.0)


@pytest.mark.parametrize("up", [24, -24, 60])
def test_halves_of_a_head_far_apart(u, up):
    rng = np.random.default_rng(3)
    k, v = rng.standard_normal((2, 150, 2, 128))
    v[..., 64:] *= 2.0 ** up
    q = torch.from_numpy(rng.standard_normal((2, 4, 128))).bfloat16()
    attend_and_check(u, "i4", q, k, v, 0.1)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("up", [-90, 100])
def test_values_of_all_magnitudes(u, kind, up):
    rng = np.random.default_rng(4)
    k, v = rng.standard_normal((2, 400, 1, 128))
    q = torch.from_numpy(rng.standard_normal((1, 2, 128))).bfloat16()
    attend_and_check(u, kind, q, k, v * 2.0 ** up, 0.1)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("n", [1, 45, 300])
@pytest.mark.parametrize("query,key,scale", [
    (-130, 0, 1e-3),  # subnormal queries: all tokens count alike
    (-130, 0, 1e-30), (0, 0, 1e-40),
    (122, None, None), (126, None, 1.0),  # keys of zero
    (122, -98, None), (125, -95, 2.0 ** -30), (120, -98, 1.0),
])
def test_queries_at_the_ends_of_their_type(u, kind, n, query, key, scale):
    """bf16 queries of 2^query, keys of 2^key (None: zeros): the scores are finite numbers, and so are the results."""
    rng = np.random.default_rng(5)
    k, v = rng.standard_normal((2, n, 1, 128))
    q = torch.from_numpy(np.clip(rng.standard_normal((2, 2, 128)), -3, 3) * 2.0 ** query).bfloat16()
    q[0, 1] = 0  # (a row of another magnitude beside it)
    attend_and_check(u, kind, q, k * 2.0 ** key if key is not None else 0 * k, v, 128 ** -0.5 if scale is None else scale)
