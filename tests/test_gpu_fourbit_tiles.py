"""Products at sizes between which every tile of tokens and rows is taken, with K whole and in parts, and with the
activations' sums made in the kernel and in a launch of their own; row and token counts end inside a tile.  Of few tokens:
every number of waves and of tiles asked for together, shares of K that they divide and do not, waves without a share."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from test_gpu_fourbit import activations, check, u, weights  # noqa: E402,F401

SIZES = [  # N, K, M
    (48, 11008, 5), (4112, 128, 5), (22032, 4096, 5), (22032, 28672, 17), (28688, 28672, 61), (32864, 28288, 83),
    (11024, 384, 93), (22032, 11008, 93), (1040, 4096, 150), (4112, 4096, 150), (6032, 8192, 150), (16400, 28672, 150),
    (6032, 8192, 250), (11024, 8192, 250), (11024, 28672, 250), (43344, 8576, 276), (28688, 128, 300), (8208, 8192, 300),
    (11024, 28672, 300), (6032, 640, 333), (6032, 8192, 333), (11024, 640, 400), (528, 8192, 400), (6032, 28672, 400),
    (8208, 640, 450), (8208, 11008, 450), (6032, 640, 500), (528, 8192, 500), (6032, 2048, 500), (6032, 11008, 500),
    (2064, 8192, 600), (1040, 4096, 900), (1040, 8192, 900), (22032, 640, 900), (6032, 8192, 900), (4112, 2048, 1100),
    (4112, 1152, 1300), (6032, 1152, 1300), (4112, 2048, 1500), (1040, 11008, 1500), (272, 28672, 2000),
    (28688, 384, 2000), (2064, 4096, 2000), (11024, 2048, 2000), (6032, 8192, 2000), (28688, 2048, 2000),
    (1040, 28672, 2300), (28688, 1152, 2300), (2064, 4096, 2600), (8208, 1152, 2600), (528, 8192, 3300),
    (28688, 2048, 3300), (1040, 1152, 5000), (10848, 9472, 94), (10832, 25984, 106)]


@pytest.mark.parametrize("kind", ["f16", "bf16", "i8"])
@pytest.mark.parametrize("N,K,M", SIZES)
def test_tiles(u, kind, N, K, M):
    codes, scales = weights(N, K, N + M)
    x = activations(M, K, kind, M)
    room = torch.full((M + 1, N), 7.0, device="cuda")  # (a row behind the last token stays as it was)
    y = u.fourbit_gemm(u.fourbit_pack(codes, scales), N, K, x, out=room[:M])
    assert (room[M] == 7).all()
    check(y, x, codes, scales)


@pytest.mark.parametrize("kind", ["f16", "bf16", "i8"])
@pytest.mark.parametrize("N", [48, 4112, 22032])
@pytest.mark.parametrize("K", [128, 640, 1152, 2048, 2560, 3584, 4608, 5120, 5632, 7168, 9216, 11008, 13824, 15360, 20480, 32768, 49152])
def test_few_tokens(u, kind, N, K):
    codes, scales = weights(N, K, N + K)
    packed = u.fourbit_pack(codes, scales)
    for M in (1, 2, 3):
        x = activations(M, K, kind, M)
        room = torch.full((M + 1, N), 7.0, device="cuda")
        y = u.fourbit_gemm(packed, N, K, x, out=room[:M])
        assert (room[M] == 7).all()
        check(y, x, codes, scales)


@pytest.mark.parametrize("kind", ["f16", "i8"])
@pytest.mark.parametrize("shapes", [[(4096, 4096)] * 3, [(16, 128), (4112, 5120), (22032, 640)], [(16, 2560)] * 8, [(8208, 1152), (48, 11008)]])
def test_few_tokens_in_batches(u, kind, shapes):
    """Batches whose problems share the workgroups out unevenly, or have fewer groups than there are waves."""
    made = [weights(N, K, i) for i, (N, K) in enumerate(shapes)]
    packed = [u.fourbit_pack(*m) for m in made]
    for M in (1, 2, 4):
        xs = {K: activations(M, K, kind, K) for _, K in shapes}
        ys = u.fourbit_gemm_batched([(p, N, K, xs[K], None) for p, (N, K) in zip(packed, shapes)], out_dtype=torch.float32)
        for y, (N, K), m in zip(ys, shapes, made):
            check(y, xs[K], *m)


@pytest.mark.parametrize("kind", ["f16", "bf16", "i8"])
@pytest.mark.parametrize("N", [272, 4096, 4112, 8192, 8208, 22032])
@pytest.mark.parametrize("K", [512, 1024, 1152, 2048, 2560, 4096, 4224, 5888, 8192, 8320, 14592, 16384, 16512])
def test_five_to_sixteen_tokens(u, kind, N, K):
    """Both sides of where one kernel takes over from another."""
    codes, scales = weights(N, K, N + K)
    packed = u.fourbit_pack(codes, scales)
    for M in (5, 8, 9, 16):
        x = activations(M, K, kind, M)
        room = torch.full((M + 1, N), 7.0, device="cuda")
        y = u.fourbit_gemm(packed, N, K, x, out=room[:M])
        assert (room[M] == 7).all()
        check(y, x, codes, scales)
