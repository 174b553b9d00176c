"""Rows of the norm and of gated activations that share memory where a call does not allow it are refused, wherever they begin
(every call fails validation, so no kernel is launched and the addresses are never read)."""
import os

import pytest

import paper_2606_10520_amd.unisvq as u

pytestmark = pytest.mark.skipif(not os.path.exists(u.LIB_PATH), reason="libunisvq.so not built")

EINVAL = -1
X, W, R, H, Y, S, G, V = (i << 24 for i in range(1, 9))  # 16 MB apart


def norm(tokens=4, n=256, x=X, xs=256, xt=u.F16, w=W, wt=u.F16, r=R, rs=256, h=H, hs=256, rt=u.F16, y=Y, ys=256, yt=u.F16, s=S):
    return u.load().unisvq_rmsnorm(tokens, n, x, xs, xt, w, wt, 0.0, 1e-5, r, rs, h, hs, rt, y, ys, yt, s, None)


def gated(tokens=4, n=256, g=G, gs=256, v=V, vs=256, y=Y, ys=256, yt=u.F16, s=S):
    return u.load().unisvq_gated(tokens, n, g, gs, v, vs, u.F16, 0, y, ys, yt, s, None)


# (rows of 512 bytes in 16 bits; four of them 2048)
@pytest.mark.parametrize("args", [
    dict(y=X + 16), dict(y=X - 16), dict(y=X + 512), dict(y=X + 1536), dict(y=X - 1536), dict(y=X + 2032), dict(y=X - 2032),
    dict(y=R + 16), dict(y=R - 512), dict(y=W + 496), dict(y=W - 2032), dict(y=H + 16), dict(y=H - 1536), dict(y=H + 2032),
    dict(h=X + 16), dict(h=X - 512), dict(h=R + 512), dict(h=R - 2032), dict(h=W + 16), dict(h=W - 2032),
    dict(rt=u.F32, h=R + 32), dict(rt=u.F32, h=R - 4080), dict(rt=u.F32, y=H + 4080), dict(yt=u.F32, y=X + 2032),
    dict(yt=u.F32, y=X - 4080), dict(yt=u.I8, y=X + 16), dict(yt=u.I8, y=X - 1008), dict(wt=u.F32, y=W + 1008),
    dict(yt=u.I8, s=X + 2044), dict(yt=u.I8, s=R - 12), dict(yt=u.I8, s=W), dict(yt=u.I8, s=H + 4), dict(yt=u.I8, s=Y + 1020),
    dict(x=X, xs=512, y=X + 496, ys=512), dict(x=X, xs=512, y=X - 496, ys=512), dict(x=X, xs=512, y=X + 1008, ys=512),
    dict(x=X, xs=512, y=X + 512 + 2048, ys=-512 + 8), dict(x=X, xs=-512, y=X + 496, ys=512), dict(x=X, xs=0, y=X + 256),
    dict(x=X, xs=1024, y=X + 2048 - 512, ys=256), dict(x=X, xs=1024, y=X + 6144 - 3 * 1024 - 496, ys=512),
    dict(x=X, xs=1024, y=X + 6144 - 3 * 528 - 496, ys=264), dict(tokens=1, y=X + 16), dict(tokens=1, y=X - 496, ys=9),
    dict(tokens=1 << 20, xs=1 << 30, y=X + (((1 << 20) - 1) << 31) - ((1 << 20) - 1 << 9) - 16),
])
def test_norm(args):
    assert norm(**args) == EINVAL


@pytest.mark.parametrize("args", [
    dict(y=G + 16), dict(y=V - 16), dict(y=G + 1536), dict(y=V - 2032), dict(yt=u.F32, y=G - 4080), dict(yt=u.I8, y=V + 2032),
    dict(yt=u.I8, s=G + 16), dict(yt=u.I8, s=V - 12), dict(yt=u.I8, s=Y + 4), dict(v=G + 512, gs=512, vs=512, y=G + 496, ys=512),
    dict(v=G + 512, gs=512, vs=512, y=G + 16, ys=512), dict(v=G + 512, gs=512, vs=512, y=G + 1024 - 16, ys=768),
    dict(gs=512, y=G + 3 * 1024 - 3 * 512 + 496, ys=256), dict(tokens=1, y=V + 496),
])
def test_gated(args):
    assert gated(**args) == EINVAL
