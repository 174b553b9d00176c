"""4-bit products of 5 to 16 tokens where the rules of sizes change kernels and variants: rows shared out in fours of tiles
(25 to 31 groups of columns), and batches, whose rows count together and whose longest rows decide."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from test_gpu_fourbit import activations, check, u, weights  # noqa: E402,F401 (u is a fixture)


@pytest.mark.parametrize("kind", ["f16", "bf16", "i8"])
@pytest.mark.parametrize("N", [4112, 8208, 18944])
@pytest.mark.parametrize("K", [2176, 3200, 3584, 3840, 3968])
def test_shares_of_any_length(u, kind, N, K):
    codes, scales = weights(N, K, N + K)
    packed = u.fourbit_pack(codes, scales)
    for M in (5, 6, 7, 8):
        x = activations(M, K, kind, M)
        room = torch.full((M + 1, N), 7.0, device="cuda")
        y = u.fourbit_gemm(packed, N, K, x, out=room[:M])
        assert (room[M] == 7).all()
        check(y, x, codes, scales)


@pytest.mark.parametrize("kind", ["f16", "bf16", "i8"])
@pytest.mark.parametrize("shapes", [
    [(11008, 4096)] * 2, [(4096, 4096), (1024, 4096), (1024, 4096)], [(3584, 3584), (512, 3584), (512, 3584)],
    [(2048, 4096), (512, 4096), (512, 4096)], [(2048, 2048), (512, 2048), (512, 2048)], [(4096, 1024), (2048, 1024), (16, 1024)],
    [(8208, 4096), (48, 384), (528, 2560)], [(2048, 1024), (528, 640), (16, 2048)], [(16, 128), (4112, 3200), (16, 128)]])
def test_batches(u, kind, shapes):
    """Gate and up, q/k/v, and problems of several K; each output in the middle of others, which stay as they are."""
    made = [weights(N, K, i) for i, (N, K) in enumerate(shapes)]
    packed = [u.fourbit_pack(*m) for m in made]
    for M in (5, 8, 9, 12, 16):
        xs = {K: activations(M, K, kind, K) for _, K in shapes}
        rooms = [torch.full((M + 2, N), 7.0, device="cuda") for N, _ in shapes]
        ys = u.fourbit_gemm_batched([(p, N, K, xs[K], r[1:-1]) for p, (N, K), r in zip(packed, shapes, rooms)])
        for y, r, (N, K), m in zip(ys, rooms, shapes, made):
            assert (r[0] == 7).all() and (r[-1] == 7).all()
            check(y, xs[K], *m)
