"""Operands of the norm and of gated activations that lie between one another's rows in one buffer, without a byte in common,
against the same calls on memory of their own."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from test_gpu_layer_rows import rows, u  # noqa: E402,F401 (u is a fixture)


@pytest.mark.parametrize("n", [64, 1000, 4096])
def test_operands_between_rows(u, n):
    M = 6
    x, r, w = rows(M, n, torch.float16, 1), rows(M, n, torch.float16, 2), rows(1, n, torch.float16, 3)[0].contiguous()
    y, h = u.rmsnorm(x, w, residual=r)
    # one stride for all: columns of a wide buffer
    b = torch.full((M, 5 * n), 7.0, dtype=torch.float16, device="cuda")
    b[:, :n], b[:, 2 * n:3 * n] = x, r
    u.rmsnorm(b[:, :n], w, residual=b[:, 2 * n:3 * n], residual_out=b[:, n:2 * n], out=b[:, 4 * n:])
    assert torch.equal(b[:, n:2 * n], h) and torch.equal(b[:, 4 * n:], y) and (b[:, 3 * n:4 * n] == 7).all()
    assert torch.equal(b[:, :n], x) and torch.equal(b[:, 2 * n:3 * n], r)
    # several strides: x in every other row, y beside all of the first ones, the weight in a gap
    b = torch.full((2 * M, 3 * n), 7.0, dtype=torch.float16, device="cuda")
    b[::2, :n], b[1, :n] = x, w
    u.rmsnorm(b[::2, :n], b[1, :n], residual=r, residual_out=b[1::2, 2 * n:], out=b[:M, n:2 * n])
    assert torch.equal(b[:M, n:2 * n], y) and torch.equal(b[1::2, 2 * n:], h) and (b[M:, n:2 * n] == 7).all()
    assert (b[::2, 2 * n:] == 7).all() and (b[3::2, :n] == 7).all()
    # gate and up as halves of fused rows, the result behind each
    g, v = rows(M, n, torch.float16, 4), rows(M, n, torch.float16, 5)
    b = torch.cat([g, v, torch.full_like(g, 7.0)], 1)
    assert torch.equal(u.gated(b[:, :n], b[:, n:2 * n], out=b[:, 2 * n:]), u.gated(g, v))
    # bytes and their scales into given tensors
    b = torch.empty((M, n), dtype=torch.int8, device="cuda"), torch.empty(M, device="cuda")
    assert all(torch.equal(p, q) for p, q in zip(u.gated(g, v, out=b), u.gated(g, v, out_dtype=torch.int8)))


def test_shifted_rows_are_refused(u):
    b = torch.zeros((9, 64), dtype=torch.float16, device="cuda")
    w = torch.ones(64, dtype=torch.float16, device="cuda")
    for call in (lambda: u.rmsnorm(b[:8], w, out=b[1:]), lambda: u.gated(b[1:], b[1:], out=b[:8]),
                 lambda: u.rmsnorm(b[:4], w, residual=b[4:8], residual_out=b[5:])):
        with pytest.raises(u.UniSVQError):
            call()
    assert not b.any()
