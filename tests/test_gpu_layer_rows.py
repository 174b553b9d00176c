"""Norm with the residual's addition and gated activations against 64-bit references, elementwise.

Tolerances.  A rounding to type T is off by eps(T) / 2 of the value, or by half of T's smallest step.  The norm's fp32
part: sums of at most 65536 squares in chains of 16 and a tree of 10 adds (26 * 2^-24, halved by the root), the root's
reciprocal (2^-23), the mean and eps (2 * 2^-24), w + offset and two products (3 * 2^-24): below 2^-19.  The gating's: its
argument t is off by 8 * 2^-24 |t|, which the exponential makes relative, and sixteen roundings are more than it has."""
import math

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

T = {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}


@pytest.fixture(scope="module")
def u():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2606_10520_amd.unisvq as u
    u.load()
    return u


def step(dtype):
    """Half a rounding, relative to the value and at least."""
    f = torch.finfo(dtype)
    return f.eps / 2, f.tiny * f.eps / 2


def rows(M, n, dtype, seed, pad=0, scale=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    t = (torch.randn((M, n + pad), generator=g, device="cuda") * scale).to(dtype)
    return t[:, :n]


def norm64(h, w, offset, eps):
    h = h.double()
    return h / (h.square().mean(1, keepdim=True) + eps).sqrt() * (w.double() + offset)


def close(y, want, rel, least=0.0):
    assert y.shape == want.shape
    off = (y.double() - want).abs()
    allowed = rel * want.abs() + least
    assert (off <= allowed).all(), f"{(off / allowed.clamp_min(1e-300)).max().item():.2f} times what is allowed"


def held(y):
    """Codes and scales that rows y (fp32) have by the rule for 8 bits.  (Divided by a tensor: a division by a number is a
    product with its reciprocal here.)"""
    a = y.abs().amax(1)
    scale = torch.where(a < 1e-30, torch.zeros_like(a), a / torch.full_like(a, 127.0))
    inv = torch.where(scale > 0, torch.ones_like(a) / scale, torch.zeros_like(a))
    return torch.round(y * inv[:, None]).to(torch.int8), scale


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("stream,weight", [("", ""), ("same", "f32"), ("f32", "")])
@pytest.mark.parametrize("M,n", [(1, 8), (33, 16), (5, 64), (70, 72), (3, 128), (9, 512), (2, 520), (300, 1000), (1, 4096),
                                 (7, 8192), (3, 8200), (4, 16384), (2, 28672), (3, 65536), (0, 4096)])
def test_norm(u, dtype, stream, weight, M, n):
    dt = T[dtype]
    x = rows(M, n, dt, M + n, pad=8 * (M % 3), scale=3.0)
    w = (1 + 0.2 * rows(1, n, torch.float32, 5)[0]).to(T.get(weight, dt))
    r = None if not stream else rows(M, n, T.get(stream, dt), 7, pad=16)
    kept = x.clone()
    y = u.rmsnorm(x, w, 1e-5, residual=r)
    h = x
    if r is not None:
        y, h = y
        assert h.dtype == r.dtype and torch.equal(h, (x.float() + r.float()).to(r.dtype))
    rel, least = step(dt)
    close(y, norm64(h, w, 0.0, 1e-5), rel + 2.0 ** -19, least)
    # the same rows in 32 and in 8 bits, the second from the first by the rule, bit for bit
    wide = u.rmsnorm(x, w, 1e-5, residual=r, out_dtype=torch.float32)
    codes = u.rmsnorm(x, w, 1e-5, residual=r, out_dtype=torch.int8)
    if r is not None:
        (wide, h1), (codes, h2) = wide, codes
        assert torch.equal(h1, h) and torch.equal(h2, h)
    close(wide, norm64(h, w, 0.0, 1e-5), 2.0 ** -19, 1e-38)
    assert torch.equal(wide.to(dt), y)
    if M:
        want, scale = held(wide)
        assert torch.equal(codes[1], scale) and torch.equal(codes[0], want)
    assert torch.equal(x, kept)


def test_norm_offset_and_eps(u):
    x, w = rows(11, 1024, torch.bfloat16, 1, scale=1e-3), rows(1, 1024, torch.bfloat16, 2, scale=0.1)[0]
    rel, least = step(torch.bfloat16)
    for eps in (1e-6, 1e-2, 3.0):
        close(u.rmsnorm(x, w, eps, weight_offset=1.0), norm64(x, w, 1.0, eps), rel + 2.0 ** -19, least)


@pytest.mark.parametrize("stream", ["f16", "f32"])
@pytest.mark.parametrize("n", [256, 4096, 20480])
def test_norm_in_place(u, stream, n):
    x, r = rows(37, n, torch.float16, 3), rows(37, n, T[stream], 4)
    w = rows(1, n, torch.float16, 5)[0].contiguous()
    y, h = u.rmsnorm(x, w, residual=r)
    a, b = x.clone(), r.clone()
    y1, h1 = u.rmsnorm(a, w, residual=b, residual_out=b, out=a)
    assert y1 is a and h1 is b and torch.equal(a, y) and torch.equal(b, h)
    if stream == "f16":  # the stream's sum in x's place, the rows in the old stream's
        a, b = x.clone(), r.clone()
        u.rmsnorm(a, w, residual=b, residual_out=a, out=b)
        assert torch.equal(a, h) and torch.equal(b, y)


@pytest.mark.parametrize("stream", ["f16", "f32"])
@pytest.mark.parametrize("n", [72, 520, 4160, 8200, 8704, 9224, 12808, 16376, 16392, 20488])
def test_norm_in_place_in_eight_bits(u, stream, n):
    """The stream written where it was read, by other waves than those that read its last run again."""
    x, r = rows(300, n, torch.float16, 3), rows(300, n, T[stream], 4)
    r[:, -8:] += 50.0  # (the sum with x twice would be the row's largest)
    x[:, -8:] += 50.0
    w = rows(1, n, torch.float16, 5)[0].abs().contiguous()
    (codes, scales), h = u.rmsnorm(x, w, residual=r, out_dtype=torch.int8)
    want = held(u.rmsnorm(x, w, residual=r, out_dtype=torch.float32)[0])
    assert torch.equal(codes, want[0]) and torch.equal(scales, want[1])
    for place in ("stream", "x") if stream == "f16" else ("stream",):
        a, b = x.clone(), r.clone()
        to = b if place == "stream" else a
        (c, s), k = u.rmsnorm(a, w, residual=b, residual_out=to, out_dtype=torch.int8)
        assert k is to and torch.equal(k, h) and torch.equal(c, codes) and torch.equal(s, scales)


def test_a_single_row_has_any_stride(u):
    x, r = (rows(4096, 1, torch.float16, i).contiguous().t() for i in (1, 2))
    assert x.shape == (1, 4096) and x.stride() == (1, 1)
    w = torch.ones(4096, dtype=torch.float16, device="cuda")
    y, h = u.rmsnorm(x, w, residual=r, residual_out=r.clone())
    want, k = u.rmsnorm(x.contiguous().view(4096).view(1, 4096), w, residual=r.reshape(4096).view(1, 4096))
    assert torch.equal(y, want) and torch.equal(h, k)
    assert torch.equal(u.gated(x, r), u.gated(x.reshape(4096).view(1, 4096), r.reshape(4096).view(1, 4096)))


def test_norm_rows_of_views_leave_the_rest(u):
    """Rows of a wider tensor, in and out; what lies between them stays."""
    big = rows(20, 640, torch.float16, 1)
    out = torch.full((20, 768), 7.0, dtype=torch.float16, device="cuda")
    w = torch.ones(256, dtype=torch.float16, device="cuda")
    u.rmsnorm(big[::2, 128:384], w, out=out[:10, 256:512])
    close(out[:10, 256:512], norm64(big[::2, 128:384], w, 0, 1e-5), 2.0 ** -11 + 2.0 ** -19, 2.0 ** -25)
    out[:10, 256:512] = 7.0
    assert (out == 7.0).all()


def test_norm_of_extreme_rows(u):
    """Zeros, values that are not finite, and the largest fp16 rows, each alone in its row."""
    x = rows(8, 1000, torch.float16, 9)
    x = x.clone()
    x[1] = 0
    x[2, 5] = math.inf
    x[3, 999] = math.nan
    x[4] = 65504.0
    x[5] = 2.0 ** -24
    w = torch.ones(1000, dtype=torch.float16, device="cuda")
    fine = [0, 1, 4, 5, 6, 7]
    y = u.rmsnorm(x, w)
    close(y[fine], norm64(x[fine], w, 0, 1e-5), 2.0 ** -11 + 2.0 ** -19, 2.0 ** -25)
    assert (y[1] == 0).all() and y[2, 5].isnan() and (y[2, :5] == 0).all() and y[3].isnan().all()
    codes, scale = u.rmsnorm(x, w, out_dtype=torch.int8)
    assert scale[1] == 0 and scale[2:4].isnan().all() and not codes[1:4].any() and scale[fine].isfinite().all()
    h = u.rmsnorm(x, w, residual=x.clone())[1]  # fp16's range is left where the sum leaves it
    assert h[4].isinf().all() and torch.equal(h[0], x[0] * 2)


def test_norm_of_more_rows_than_workgroups(u):
    M, n = (1 << 20) + 3, 520
    x = torch.empty((M, n), dtype=torch.float16, device="cuda").normal_()
    w = torch.ones(n, dtype=torch.float16, device="cuda")
    y = u.rmsnorm(x, w)
    for part in (slice(0, 4), slice((1 << 20) - 2, M)):
        close(y[part], norm64(x[part], w, 0, 1e-5), 2.0 ** -11 + 2.0 ** -19, 2.0 ** -25)


def test_norm_past_32_bit_offsets(u):
    """Row strides that put the last rows past 2^32 elements."""
    store = torch.zeros((1 << 32) + (1 << 20), dtype=torch.float16, device="cuda")
    x = store.as_strided((3, 4096), (1 << 31, 1))
    x.copy_(rows(3, 4096, torch.float16, 1))
    w = torch.ones(4096, dtype=torch.float16, device="cuda")
    assert torch.equal(u.rmsnorm(x, w), u.rmsnorm(x.contiguous(), w))
    assert torch.equal(u.gated(x, x), u.gated(x.contiguous(), x.contiguous()))


def gate64(g, v, act):
    g, v = g.double(), v.double()
    t = g if act == "silu" else math.sqrt(8 / math.pi) * (g + 0.044715 * g ** 3)
    return g * v / (1 + torch.exp(-t)), t


def check_gated(y, g, v, act, dtype):
    want, t = gate64(g, v, act)
    rel, least = step(dtype)
    # (where exp(-t) passes fp32's range the result is zero: what is lost is below 1e-38 of g v)
    allowed = (rel + (8 * t.abs().clamp_max(120) + 16) * 2.0 ** -24) * want.abs() + least + 1e-36 * (g.double() * v.double()).abs()
    assert ((y.double() - want).abs() <= allowed).all()


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("act", ["silu", "gelu"])
@pytest.mark.parametrize("M,n", [(1, 8), (3, 72), (33, 1000), (1, 11008), (5, 28672), (2, 65536), (0, 64)])
def test_gated(u, dtype, act, M, n):
    dt = T[dtype]
    both = rows(M, 2 * n, dt, M + n, scale=4.0)
    g, v = both[:, :n], both[:, n:]  # the halves of one fused row
    y = u.gated(g, v, act)
    check_gated(y, g, v, act, dt)
    wide = u.gated(g, v, act, out_dtype=torch.float32)
    check_gated(wide, g, v, act, torch.float32)
    assert torch.equal(wide.to(dt), y)
    codes, scale = u.gated(g, v, act, out_dtype=torch.int8)
    if M:
        want, top = held(wide)
        assert torch.equal(scale, top) and torch.equal(codes, want)
    flat = u.gated(g.contiguous(), v.contiguous(), act)
    assert torch.equal(flat, y)


@pytest.mark.parametrize("act", ["silu", "gelu"])
def test_gated_over_the_whole_range(u, act):
    """Every finite fp16 as a gate, and bf16 gates of any magnitude."""
    g = torch.arange(1 << 16, device="cuda", dtype=torch.int32).to(torch.int16).view(torch.float16).view(64, 1024)
    g = torch.where(g.isfinite(), g, torch.zeros_like(g))
    one = torch.ones_like(g)
    check_gated(u.gated(g, one, act), g, one, act, torch.float16)
    b = torch.arange(0, 1 << 16, device="cuda", dtype=torch.int32).to(torch.int16).view(torch.bfloat16).view(64, 1024)
    b = torch.where(b.abs() < 1e12, b, torch.zeros_like(b))
    one = torch.ones_like(b)
    check_gated(u.gated(b, one, act), b, one, act, torch.bfloat16)


def test_gated_in_place_and_not_finite(u):
    g, v = rows(9, 520, torch.float16, 1), rows(9, 520, torch.float16, 2)
    want = u.gated(g, v)
    a, b = g.clone(), v.clone()
    assert u.gated(a, v, out=a) is a and torch.equal(a, want)
    assert torch.equal(u.gated(g, b, out=b), want)
    g = g.clone()
    g[3, 7] = math.inf
    g[4, 8] = math.nan
    y = u.gated(g, v.abs() + 1)
    assert y[3, 7] == math.inf and y[4, 8].isnan() and y.isfinite().sum() == 9 * 520 - 2
    codes, scale = u.gated(g, v, out_dtype=torch.int8)
    assert scale[3:5].isnan().all() and not codes[3:5].any()
    fine = [0, 1, 2, 5, 6, 7, 8]
    assert torch.equal(codes[fine], u.gated(g[fine].contiguous(), v[fine], out_dtype=torch.int8)[0])


def test_rows_on_another_stream(u):
    s = torch.cuda.Stream()
    x, w = rows(64, 4096, torch.float16, 1), torch.ones(4096, dtype=torch.float16, device="cuda")
    torch.cuda.synchronize()
    y = u.rmsnorm(x, w, stream=s)
    z = u.gated(y, x, stream=s, out_dtype=torch.int8)
    s.synchronize()
    assert torch.equal(y, u.rmsnorm(x, w)) and torch.equal(z[0], u.gated(y, x, out_dtype=torch.int8)[0])
