"""4-bit weights: packing, rounding, and products of 16- and 8-bit activations against 64-bit references, elementwise.

Tolerance of a product.  Codes are exact operands.  Of 16-bit activations a group's sum is eight products of the matrix
cores (four of them with -8), each off by at most 2 * 2^-24 of the magnitudes summed so far, m_g = sum |x| (c + 8); of
8-bit ones it is exact.  The groups' sums are multiplied and added in fp32, at most groups + 40 roundings (waves, and parts
of a long K), and y is rounded once."""
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


def weights(N, K, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    codes = torch.randint(0, 16, (N, K), generator=g, device="cuda", dtype=torch.uint8)
    scales = ((torch.rand((N, K // 128), generator=g, device="cuda") + 0.2) * 0.02).half()
    return codes, scales


def activations(M, K, kind, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    if kind == "i8":
        return (torch.randint(-127, 128, (M, K), generator=g, device="cuda").to(torch.int8),
                torch.rand(M, generator=g, device="cuda") + 0.1)
    x = torch.randn((M, K), generator=g, device="cuda")
    x[:, torch.rand(K, generator=g, device="cuda") < 0.01] *= 20
    return x.to(T[kind])


def check(y, x, codes, scales, at=slice(None)):
    """y against x W^T; `at`: the tokens looked at."""
    pair = isinstance(x, tuple)
    v = (x[0].double() * x[1].double()[:, None] if pair else x.double())[at]
    K = codes.shape[1]
    w = (codes.double() - 8).view(*scales.shape, 128) * scales.double()[..., None]
    want = v @ w.view(-1, K).T
    if pair:
        most = v.abs() @ w.abs().view(-1, K).T
        steps = K // 128 + 42
    else:
        most = v.abs() @ ((codes.double() + 8).view(*scales.shape, 128) * scales.double()[..., None]).view(-1, K).T
        steps = 16 + K // 128 + 40
    f = torch.finfo(y.dtype)
    allowed = steps * 2.0 ** -24 * most + f.eps / 2 * want.abs() + f.tiny * f.eps / 2
    off = (y[at].double() - want).abs()
    assert (off <= allowed).all(), f"{(off / allowed).max().item():.2f} times what is allowed"


@pytest.mark.parametrize("N,K", [(16, 128), (48, 384), (32, 512), (64, 640), (160, 1152)])
def test_pack_and_unpack(u, N, K):
    codes, scales = weights(N, K, N + K)
    bad = torch.zeros(1, dtype=torch.int32, device="cuda")
    packed = u.fourbit_pack(codes, scales, bad_codes=bad)
    groups, quads = K // 128, -(-(K // 128) // 4)
    assert packed.numel() == u.fourbit_bytes(N, K) == N * K // 2 + N * 8 * quads and bad.item() == 0
    a, b = u.fourbit_unpack(packed, N, K)
    assert torch.equal(a, codes) and torch.equal(b.view(torch.int16), scales.view(torch.int16))
    # the layout, place by place
    p, c = packed.cpu(), codes.cpu()
    for row, col in ((0, 0), (N - 1, K - 1), (N // 2, K // 2 + 21), (5, 76), (15, 4), (7, 127)):
        g, k = divmod(col, 128)
        word, slot = 2 * (k // 64) + k % 16 // 8, 16 * (k % 64 // 16) + row % 16
        byte = p[((row // 16 * groups + g) * 64 + slot) * 16 + 4 * word + k % 4].item()
        assert (byte >> 4 * (k % 8 // 4) & 15) == c[row, col]
        at = N * K // 2 + (row // 16 * quads + g // 4) * 128 + row % 16 * 8 + g % 4 * 2
        assert torch.equal(p[at:at + 2].view(torch.int16), scales.cpu()[row, g].view(1).view(torch.int16))
    codes[0, 5] = 16
    codes[N - 1, 1] = 255
    again = u.fourbit_pack(codes, scales, bad_codes=bad)
    assert bad.item() == 2 and torch.equal(u.fourbit_unpack(again, N, K)[0], codes & 15)


@pytest.mark.parametrize("dtype", ["f16", "bf16", "f32"])
@pytest.mark.parametrize("N,K", [(16, 128), (48, 640), (256, 4096)])
def test_quantize(u, dtype, N, K):
    g = torch.Generator(device="cuda").manual_seed(N)
    W = (torch.randn((N, K), generator=g, device="cuda") * 0.05).to(T[dtype])
    W[1, :128] = 0
    W[2, 3] = math.inf
    W[3, 127] = math.nan
    W[4, :128] = 1e-9 if dtype != "f16" else 0
    W[5, 7] = 6e4
    W[6, :128] = torch.arange(128, device="cuda").to(W.dtype) / 2 - 24.5  # a scale of 5.5625 and ties
    codes, scales = u.fourbit_unpack(u.fourbit_quantize(W), N, K)
    w = W.float().view(N, K // 128, 128)
    top = w.abs().amax(2)
    bad = ~w.isfinite().all(2)
    want = torch.where(bad, torch.full_like(top, math.nan), (top / torch.full_like(top, 7.0)).clamp_max(65504.0)).half()
    assert torch.equal(torch.isnan(scales), bad) and torch.equal(scales[~bad], want[~bad])
    s = want.float()[..., None]
    c = torch.where(s > 0, torch.round(w / s).clamp(-8, 7), torch.zeros_like(w)).nan_to_num(0.0) + 8
    assert torch.equal(codes, c.view(N, K).to(torch.uint8))


@pytest.mark.parametrize("kind", ["f16", "bf16", "i8"])
def test_unit_rows_give_the_weights(u, kind):
    """Products of unit vectors are the weights themselves, exactly."""
    N, K = 48, 640
    codes, scales = weights(N, K, 1)
    packed = u.fourbit_pack(codes, scales)
    w = (codes.float() - 8).view(N, K // 128, 128) * scales.float()[..., None]
    eye = torch.eye(K, device="cuda")
    x = (eye.to(torch.int8), torch.ones(K, device="cuda")) if kind == "i8" else eye.to(T[kind])
    for M in (1, 7, 40, 200, 640):
        part = (x[0][-M:].contiguous(), x[1][-M:].contiguous()) if kind == "i8" else x[-M:].contiguous()
        y = u.fourbit_gemm(packed, N, K, part, out_dtype=torch.float32)
        assert torch.equal(y, w.view(N, K).T[-M:]), M


@pytest.mark.parametrize("kind", ["f16", "bf16", "i8"])
@pytest.mark.parametrize("N,K", [(16, 128), (48, 384), (272, 640), (1040, 1152), (4096, 1024), (32, 8192)])
@pytest.mark.parametrize("M", [1, 2, 4, 5, 16, 17, 32, 33, 64, 65, 127, 129, 257, 333])
def test_product(u, kind, N, K, M):
    codes, scales = weights(N, K, N + K)
    x = activations(M, K, kind, M)
    packed = u.fourbit_pack(codes, scales)
    y = u.fourbit_gemm(packed, N, K, x, out_dtype=torch.float32)
    check(y, x, codes, scales)
    for dt in (torch.float16, torch.bfloat16):
        assert torch.equal(u.fourbit_gemm(packed, N, K, x, out_dtype=dt), y.to(dt))


@pytest.mark.parametrize("kind", ["f16", "bf16", "i8"])
@pytest.mark.parametrize("N,K,M", [(4096, 4096, 1), (4096, 11008, 3), (11008, 4096, 61), (1024, 8192, 130),
                                   (8192, 28672, 16), (4096, 4096, 1030), (11008, 4096, 512), (528, 4096, 2500)])
def test_product_at_decoder_sizes(u, kind, N, K, M):
    codes, scales = weights(N, K, N + K)
    x = activations(M, K, kind, M)
    y = u.fourbit_gemm(u.fourbit_pack(codes, scales), N, K, x, out_dtype=torch.float32)
    check(y, x, codes, scales)


@pytest.mark.parametrize("kind", ["f16", "bf16", "i8"])
@pytest.mark.parametrize("M", [1, 4, 16, 50, 70, 300])
def test_batched_products(u, kind, M):
    """Problems of different N and K, and of one x; each as a single call gives it up to the order of its sums."""
    shapes = [(4096, 512), (16, 128), (528, 512), (1024, 2048)]
    made = [weights(N, K, N) for N, K in shapes]
    xs = {K: activations(M, K, kind, K) for _, K in shapes}
    packed = [u.fourbit_pack(*m) for m in made]
    outs = [None, torch.full((M, 16), 5.0, device="cuda"), None, None]
    ys = u.fourbit_gemm_batched([(p, N, K, xs[K], o) for p, (N, K), o in zip(packed, shapes, outs)], out_dtype=torch.float32)
    assert ys[1] is outs[1]
    for y, (N, K), m in zip(ys, shapes, made):
        check(y, xs[K], *m)
    again = u.fourbit_gemm_batched([(p, N, K, xs[K], None) for p, (N, K) in zip(packed, shapes)], out_dtype=torch.float32)
    assert all(torch.equal(a, b) for a, b in zip(ys, again))


@pytest.mark.parametrize("kind", ["f16", "bf16", "i8"])
@pytest.mark.parametrize("M", [3, 16, 40, 100, 300])
def test_a_token_that_is_not_finite_stays_alone(u, kind, M):
    N, K = 272, 640
    codes, scales = weights(N, K, 3)
    packed = u.fourbit_pack(codes, scales)
    x = activations(M, K, kind, 4)
    y = u.fourbit_gemm(packed, N, K, x, out_dtype=torch.float32)
    if kind == "i8":
        x[1][1] = math.nan
        x[1][2] = 0.0
    else:
        x[1, 5] = math.inf
        x[2, K - 1] = math.nan
    z = u.fourbit_gemm(packed, N, K, x, out_dtype=torch.float32)
    rest = [t for t in range(M) if t not in (1, 2)]
    assert z[1].isnan().all() and torch.equal(z[rest], y[rest])
    assert not z[2].any() if kind == "i8" else z[2].isnan().all()


@pytest.mark.parametrize("kind", ["f16", "bf16"])
def test_large_and_small_activations(u, kind):
    """The whole range of the type: its largest values with codes 0 and 15, and its subnormals."""
    N, K = 32, 256
    codes, scales = weights(N, K, 3)
    codes[:16], codes[16:] = 0, 15
    top = 65504.0 if kind == "f16" else 2.0 ** 100
    x = torch.stack([torch.full((K,), top), torch.full((K,), 2.0 ** -24 if kind == "f16" else 2.0 ** -100)]).cuda().to(T[kind])
    check(u.fourbit_gemm(u.fourbit_pack(codes, scales), N, K, x, out_dtype=torch.float32), x, codes, scales)


def test_outputs_where_they_are_not_aligned(u):
    """y needs its element's alignment alone."""
    N, K, M = 64, 256, 70
    codes, scales = weights(N, K, 1)
    packed = u.fourbit_pack(codes, scales)
    for M in (3, 70, 300):
        x = activations(M, K, "bf16", 2)
        store = torch.full((M * N + 3,), 9.0, dtype=torch.bfloat16, device="cuda")
        out = store[1:1 + M * N].view(M, N)
        u.fourbit_gemm(packed, N, K, x, out=out)
        assert torch.equal(out, u.fourbit_gemm(packed, N, K, x))
        assert store[0] == 9 and (store[1 + M * N:] == 9).all()


@pytest.mark.parametrize("M", [1, 40, 300])
def test_memory_behind_the_inputs_is_not_read_into_results(u, M):
    """x and the packed weights in the middle of NaN: nothing of it reaches y."""
    N, K = 144, 640
    codes, scales = weights(N, K, 1)
    x = activations(M, K, "f16", 2)
    packed = u.fourbit_pack(codes, scales)
    want = u.fourbit_gemm(packed, N, K, x)
    room = torch.full((M * K + 4096,), math.nan, dtype=torch.float16, device="cuda")
    room[1024:1024 + M * K] = x.view(-1)
    store = torch.full((packed.numel() + 8192,), 0xff, dtype=torch.uint8, device="cuda")
    store[4096:4096 + packed.numel()] = packed
    assert torch.equal(u.fourbit_gemm(store[4096:4096 + packed.numel()], N, K, room[1024:1024 + M * K].view(M, K)), want)


@pytest.mark.parametrize("M", [1, 16, 50, 333])
@pytest.mark.parametrize("bits", [16, 8])
def test_a_layer_in_a_graph(u, M, bits):
    """Norm, products, gating and the down product together, as a layer's feed-forward half uses them: captured once,
    replayed on new inputs between eager calls, against eager results; and every step's results against its definition
    on what the step before it gave."""
    K, F = 512, 1152
    kept = torch.float16 if bits == 16 else torch.int8
    made = [weights(F, K, 1), weights(F, K, 2), weights(K, F, 3)]
    wg, wu, wd = (u.fourbit_pack(*m) for m in made)
    w = (1 + 0.1 * torch.randn(K, device="cuda")).half()
    x, r = (torch.empty((M, K), dtype=torch.float16, device="cuda") for _ in range(2))

    def layer():
        y, h = u.rmsnorm(x, w, residual=r, out_dtype=kept)
        g, v = u.fourbit_gemm_batched([(wg, F, K, y, None), (wu, F, K, y, None)], out_dtype=torch.float16)
        a = u.gated(g, v, out_dtype=kept)
        return h, y, g, v, a, u.fourbit_gemm(wd, K, F, a, out_dtype=torch.float16)

    def parts(t):
        return t if isinstance(t, tuple) else (t,)

    x.normal_(), r.normal_()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        layer()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = layer()
    for _ in range(4):
        x.normal_(), r.normal_()
        eager = layer()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for s, t in zip(got, eager) for a, b in zip(parts(s), parts(t)))
        h, y, g, v, a, out = got
        assert torch.equal(h, (x.float() + r.float()).half())
        f = h.double()
        f = f / (f.square().mean(1, keepdim=True) + 1e-5).sqrt() * w.double()
        gate = g.double() * torch.sigmoid(g.double()) * v.double()
        for t, want in ((y, f), (a, gate)):
            # a rounding to fp16, or to codes: half a step of a row's scale; 2^-18 and 20 * 2^-24 |g| for what comes before
            value = t[0].double() * t[1].double()[:, None] if bits == 8 else t.double()
            half = t[1].double()[:, None] * 0.5 if bits == 8 else 2.0 ** -11 * want.abs() + 2.0 ** -25
            top = want.abs().amax(1, keepdim=True) if bits == 8 else want.abs()
            assert ((value - want).abs() <= half + (2.0 ** -17 + 20 * 2.0 ** -24 * g.double().abs().max()) * top).all()
        check(g, y, *made[0])
        check(v, y, *made[1])
        check(out, a, *made[2])
