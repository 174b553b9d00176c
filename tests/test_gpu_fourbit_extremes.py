"""4-bit products at the ends of their ranges: K of 2^20, weights and outputs and activations past 2^31 bytes and elements,
calls on several streams at once, captured ones that share a workspace, given outputs and workspaces."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from test_gpu_fourbit import T, activations, check, u, weights  # noqa: E402,F401 (u is a fixture)


def sliced(x, rows):
    return (x[0][rows], x[1][rows]) if isinstance(x, tuple) else x[rows]


@pytest.mark.parametrize("kind", ["bf16", "i8"])
@pytest.mark.parametrize("K,M", [(1 << 20, 1), (1 << 20, 3), (1 << 20, 16), (1 << 20, 70), ((1 << 17) + 128, 2), ((1 << 17) + 128, 130),
                                 (28672, 2), (28672, 4), (36864, 1), (72192, 1)])
def test_long_rows(u, kind, K, M):
    N = 32
    codes, scales = weights(N, K, 1)
    x = activations(M, K, kind, 2)
    check(u.fourbit_gemm(u.fourbit_pack(codes, scales), N, K, x, out_dtype=torch.float32), x, codes, scales)


@pytest.mark.parametrize("M", [1, 4, 9, 40, 200])
def test_weights_past_32_bits(u, M):
    """2.3 GB of codes: the first and the last rows are those of their own packed weights."""
    N, K = 288_000, 16384
    size = u.fourbit_bytes(N, K)
    packed = torch.randint(0, 256, (N * K // 2,), dtype=torch.uint8, device="cuda")
    packed = torch.cat([packed, torch.empty((size - N * K // 2) // 2, dtype=torch.float16, device="cuda").uniform_(0.01, 0.02).view(torch.uint8)])
    x = activations(M, K, "f16", 3)
    y = u.fourbit_gemm(packed, N, K, x, out_dtype=torch.float32)
    rows, block, quads = 64, 16 * K // 2, K // 512
    for first in (0, N - rows):
        b = first // 16
        part = torch.cat([packed[b * block:(b + rows // 16) * block], packed[N * K // 2 + b * quads * 128:][:rows // 16 * quads * 128]])
        check(y[:, first:first + rows], x, *u.fourbit_unpack(part, rows, K))


def test_outputs_past_32_bits(u):
    """More than 2^31 outputs: the first and last tokens."""
    N, K, M = 131072, 128, 16500
    codes, scales = weights(N, K, 1)
    x = activations(M, K, "bf16", 2)
    y = u.fourbit_gemm(u.fourbit_pack(codes, scales), N, K, x)
    for at in (slice(0, 2), slice(M - 2, M)):
        check(y[at], sliced(x, at), codes, scales)


@pytest.mark.parametrize("kind", ["f16", "i8"])
def test_activations_past_32_bits(u, kind):
    """More than 2^31 activations: tokens on both sides of the border and the last ones."""
    N, K = 32, 1152
    M = (1 << 31) // K + 70
    codes, scales = weights(N, K, 1)
    if kind == "i8":
        x = torch.empty((M, K), dtype=torch.int8, device="cuda").random_(-127, 128), torch.full((M,), 0.5, device="cuda")
    else:
        x = torch.empty((M, K), dtype=torch.float16, device="cuda").normal_()
    y = u.fourbit_gemm(u.fourbit_pack(codes, scales), N, K, x, out_dtype=torch.float32)
    for at in (slice(0, 3), slice(M - 75, M)):
        check(y[at], sliced(x, at), codes, scales)


@pytest.mark.parametrize("kind", ["f16", "i8"])
def test_streams_side_by_side(u, kind):
    """Calls on two streams at once, with memory of their own, again and again."""
    made = [weights(N, K, N) for N, K in ((4096, 2048), (1040, 4096))]
    packed = [u.fourbit_pack(*m) for m in made]
    cases = [(p, *m[0].shape, activations(M, m[0].shape[1], kind, M)) for p, m in zip(packed, made) for M in (1, 16, 60, 300)]
    want = [u.fourbit_gemm(*c, out_dtype=torch.float32) for c in cases]
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    for _ in range(3):
        got = [[u.fourbit_gemm(*c, out_dtype=torch.float32, stream=s) for c in (cases if i else cases[::-1])] for i, s in enumerate(streams)]
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got[1], want)) and all(torch.equal(a, b) for a, b in zip(got[0], want[::-1]))


def test_two_graphs_share_a_workspace(u):
    """Two captured calls with one workspace, replayed in turn with an eager call of a third shape between them."""
    shapes = [(1024, 8192, 40), (528, 4096, 200), (2048, 4096, 100)]
    made = [weights(N, K, N) for N, K, _ in shapes]
    packed = [u.fourbit_pack(*m) for m in made]
    xs = [activations(M, K, "bf16", M) for _, K, M in shapes]
    size = max(u.fourbit_gemm_workspace_bytes(N, K, M, torch.bfloat16) for N, K, M in shapes)
    assert size
    ws = torch.full((size,), 0xff, dtype=torch.uint8, device="cuda")
    outs = [torch.empty((M, N), dtype=torch.float32, device="cuda") for N, _, M in shapes]

    def call(i):
        N, K, _ = shapes[i]
        return u.fourbit_gemm(packed[i], N, K, xs[i], out=outs[i], workspace=ws)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        call(0), call(1)
    torch.cuda.current_stream().wait_stream(side)
    graphs = [torch.cuda.CUDAGraph() for _ in range(2)]
    for i, g in enumerate(graphs):
        with torch.cuda.graph(g):
            call(i)
    for turn in range(3):
        for x in xs:
            x.normal_()
        for o in outs:
            o.fill_(7.0)
        for i in (0, 1) if turn % 2 else (1, 0):
            graphs[i].replay()
            call(2)
        torch.cuda.synchronize()
        for o, x, m in zip(outs, xs, made):
            check(o, x, *m)


@pytest.mark.parametrize("kind", ["f16", "bf16", "i8"])
def test_exactly_the_workspace_and_nothing_behind_it(u, kind):
    """A workspace of exactly the stated bytes, in the middle of others that stay as they are; and outputs in the middle of others."""
    for N, K, M in ((1024, 8192, 40), (4096, 4096, 61), (528, 4096, 200), (272, 1152, 333), (8192, 28672, 16)):
        codes, scales = weights(N, K, N)
        x = activations(M, K, kind, M)
        size = u.fourbit_gemm_workspace_bytes(N, K, M, torch.int8 if kind == "i8" else T[kind])
        store = torch.full((size + 8192,), 0x5a, dtype=torch.uint8, device="cuda")
        room = torch.full((M + 2, N), 3.0, dtype=torch.float32, device="cuda")
        u.fourbit_gemm(u.fourbit_pack(codes, scales), N, K, x, out=room[1:-1], workspace=store[4096:4096 + size] if size else None)
        check(room[1:-1], x, codes, scales)
        assert (room[0] == 3).all() and (room[-1] == 3).all()
        assert (store[:4096] == 0x5a).all() and (store[4096 + size:] == 0x5a).all()


@pytest.mark.parametrize("kind", ["f16", "i8"])
@pytest.mark.parametrize("M", [1, 3, 12, 33, 500])
def test_the_largest_batch(u, kind, M):
    """Eight problems, more and fewer rows than a workgroup has, K from one group on."""
    shapes = [(16, 128), (32, 256), (4096, 128), (48, 1152), (1040, 640), (16, 4096), (272, 384), (64, 512)]
    made = [weights(N, K, N + K) for N, K in shapes]
    xs = [activations(M, K, kind, i) for i, (_, K) in enumerate(shapes)]
    ys = u.fourbit_gemm_batched([(u.fourbit_pack(*m), N, K, x, None) for m, (N, K), x in zip(made, shapes, xs)], out_dtype=torch.float32)
    for y, x, m in zip(ys, xs, made):
        check(y, x, *m)


def test_weights_of_zero_scale_and_of_scales_that_are_not_finite(u):
    """A scale that is not finite spoils its own row alone; zero scales give zeros."""
    N, K = 48, 640
    for M in (1, 10, 100):
        codes, scales = weights(N, K, 5)
        x = activations(M, K, "f16", M)
        want = u.fourbit_gemm(u.fourbit_pack(codes, scales), N, K, x, out_dtype=torch.float32)
        scales[7] = 0
        scales[20, 3] = float("nan")
        y = u.fourbit_gemm(u.fourbit_pack(codes, scales), N, K, x, out_dtype=torch.float32)
        rest = [r for r in range(N) if r not in (7, 20)]
        assert torch.equal(y[:, rest], want[:, rest]) and not y[:, 7].any() and y[:, 20].isnan().all()
