"""Gated activations of every finite bf16 gate, past the magnitudes at which gelu's cubic and exp(-t) leave fp32's range.

From 128 on the logistic function is 1 in fp32 (exp(-128) is below 2^-184) and the reciprocal of 1 off by an ulp at most, so
y is g u, in fp32 to three roundings; to -128 it is at most 128 exp(-128), which the entry point may take as 0 and fp32 does
not hold.  In between |t| is at most 2^17 for gelu, and where exp(-t) passes fp32's range y is 0."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from test_gpu_layer_rows import check_gated, u  # noqa: E402,F401 (u is a fixture)


@pytest.mark.parametrize("act", ["silu", "gelu"])
@pytest.mark.parametrize("up", [1.0, -0.5])
def test_every_finite_gate(u, act, up):
    g = torch.arange(1 << 16, device="cuda", dtype=torch.int32).to(torch.int16).view(torch.bfloat16)
    g = g[g.isfinite()].view(255, 256)
    v = torch.full_like(g, up)
    large, small = g >= 128, g <= -128
    between = ~(large | small)
    for dtype in (torch.bfloat16, torch.float32):
        y = u.gated(g, v, act, out_dtype=dtype)
        check_gated(y[between], g[between], v[between], act, dtype)
        want = g.double() * up
        assert ((y.double() - want).abs()[large] <= 3 * 2.0 ** -24 * want.abs()[large]).all()
        assert (y[small] == 0).all()
    codes, scale = u.gated(g, v, act, out_dtype=torch.int8)
    top = u.gated(g, v, act, out_dtype=torch.float32)
    a = top.abs().amax(1)
    assert torch.equal(scale, torch.where(a < 1e-30, torch.zeros_like(a), a / torch.full_like(a, 127.0)))
    inv = torch.where(scale > 0, torch.ones_like(a) / scale, torch.zeros_like(a))
    assert torch.equal(codes, torch.round(top * inv[:, None]).to(torch.int8))
