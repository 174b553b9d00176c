"""Refusals of the attention block's entry points: every call fails validation (or has nothing to do), so no kernel is
ever launched and the addresses are never read."""
import ctypes
import os

import pytest

import paper_2606_10520_amd.unisvq as u

pytestmark = pytest.mark.skipif(not os.path.exists(u.LIB_PATH), reason="libunisvq.so not built")

OK, EINVAL, EUNSUP, EALIGN, EWS = 0, -1, -3, -4, -6
GOOD = 0x10000
NAN, INF = float("nan"), float("inf")


def table(positions=64, rot=128, theta=1e4, factor=1.0, low=1.0, high=4.0, original=0.0, magnitude=1.0, out=GOOD):
    return u.load().unisvq_rope_table(positions, rot, theta, factor, low, high, original, magnitude, out, None)


@pytest.mark.parametrize("args,want", [
    (dict(out=None), EINVAL), (dict(positions=0), EINVAL), (dict(positions=1 << 25), EINVAL), (dict(rot=3), EINVAL),
    (dict(rot=0), EINVAL), (dict(rot=1026), EINVAL), (dict(theta=0.0), EINVAL), (dict(theta=NAN), EINVAL),
    (dict(factor=-1.0), EINVAL), (dict(factor=INF), EINVAL), (dict(original=-1.0), EINVAL),
    (dict(original=10.0, low=4.0, high=4.0), EINVAL), (dict(original=10.0, high=NAN), EINVAL),
    (dict(magnitude=NAN), EINVAL), (dict(out=GOOD + 4), EALIGN),
])
def test_rope_table_refusals(args, want):
    assert table(**args) == want


def rope(tokens=4, heads=2, D=128, rot=128, x=GOOD, xt=256, xh=128, pos=GOOD, table=GOOD, n=64, y=GOOD, yt=256, yh=128,
         dt=u.F16):
    return u.load().unisvq_rope(tokens, heads, D, rot, 0, 0, x, xt, xh, pos, table, n, y, yt, yh, dt, None)


@pytest.mark.parametrize("args,want", [
    (dict(x=None), EINVAL), (dict(y=None), EINVAL), (dict(pos=None), EINVAL), (dict(table=None), EINVAL),
    (dict(tokens=-1), EINVAL), (dict(heads=0), EINVAL), (dict(n=0), EINVAL), (dict(dt=u.F32), EINVAL),
    (dict(dt=9), EINVAL), (dict(D=120), EUNSUP), (dict(D=0), EUNSUP), (dict(D=1040), EUNSUP), (dict(rot=136), EUNSUP),
    (dict(rot=24), EUNSUP), (dict(rot=0), EUNSUP), (dict(rot=144), EUNSUP), (dict(tokens=1 << 31), EUNSUP),
    (dict(tokens=1 << 30, heads=2), EUNSUP), (dict(x=GOOD + 2), EALIGN), (dict(xt=257), EALIGN), (dict(yh=4), EALIGN),
    (dict(y=GOOD + 8), EALIGN), (dict(table=GOOD + 4), EALIGN), (dict(pos=GOOD + 2), EALIGN), (dict(tokens=0), OK),
])
def test_rope_refusals(args, want):
    assert rope(**args) == want


def cache(pages=8, page=64, heads=2, D=128, kind=u.CACHE_I8, k=GOOD, v=GOOD, ks=GOOD, vs=GOOD):
    return u.Cache(pages, page, heads, D, kind, k, v, ks, vs)


def append(c=None, pt=GOOD, B=2, width=4, tokens=3, seqs=GOOD, pos=GOOD, k=GOOD, kt=256, v=GOOD, vh=128, q=GOOD, qh=4,
           qo=GOOD, dt=u.F16, table=GOOD, n=64, rot=128):
    return u.load().unisvq_cache_append(c or cache(), pt, B, width, tokens, seqs, pos, k, kt, 128, v, 256, vh, q, qh, 512,
                                        128, qo, 512, 128, dt, table, n, rot, 0, None)


def read(c=None, pt=GOOD, B=2, width=4, starts=None, cu=GOOD, tokens=3, k=GOOD, kt=256, v=GOOD, dt=u.F16):
    return u.load().unisvq_cache_read(c or cache(), pt, B, width, starts, cu, tokens, k, kt, 128, v, 256, 128, dt, None)


def decode(c=None, pt=GOOD, B=2, width=4, lens=GOOD, max_len=0, q_len=1, qh=4, q=GOOD, qt=512, dt=u.F16, scale=0.1,
           out=GOOD, ot=512, lse=None, ws=GOOD, size=1 << 40):
    return u.load().unisvq_attn_decode(c or cache(), pt, B, width, lens, max_len, q_len, qh, q, qt, 128, dt, scale, out,
                                       ot, 128, lse, ws, size, None)


BAD_CACHES = [
    (dict(kind=4), EINVAL), (dict(kind=-1), EINVAL), (dict(pages=0), EINVAL), (dict(pages=1 << 31), EINVAL),
    (dict(heads=0), EINVAL), (dict(heads=70000), EINVAL), (dict(page=8), EUNSUP), (dict(page=48), EUNSUP),
    (dict(page=512), EUNSUP), (dict(D=96), EUNSUP), (dict(k=None), EINVAL), (dict(v=None), EINVAL),
    (dict(ks=None), EINVAL), (dict(vs=None), EINVAL), (dict(k=GOOD + 8), EALIGN), (dict(vs=GOOD + 4), EALIGN),
    (dict(kind=u.CACHE_I4, ks=None), EINVAL),
]


@pytest.mark.parametrize("call", [append, read, decode])
@pytest.mark.parametrize("args,want", BAD_CACHES)
def test_cache_refusals(call, args, want):
    assert call(c=cache(**args)) == want


@pytest.mark.parametrize("call", [append, read, decode])
def test_page_table_refusals(call):
    assert call(pt=None) == EINVAL
    assert call(B=-1) == EINVAL
    assert call(width=-1) == EINVAL
    assert call(pt=GOOD + 1) == EALIGN
    assert call(width=1 << 25) == EUNSUP  # more tokens than positions count


@pytest.mark.parametrize("args,want", [
    (dict(tokens=-1), EINVAL), (dict(pos=None), EINVAL), (dict(k=None), EINVAL), (dict(v=None), EINVAL),
    (dict(q=None), EINVAL), (dict(qo=None), EINVAL), (dict(qh=-1), EINVAL), (dict(dt=u.F32), EINVAL),
    (dict(n=0), EINVAL), (dict(rot=40), EUNSUP), (dict(rot=256), EUNSUP), (dict(kt=12), EALIGN), (dict(vh=4), EALIGN),
    (dict(k=GOOD + 2), EALIGN), (dict(q=GOOD + 8), EALIGN), (dict(seqs=GOOD + 2), EALIGN), (dict(table=GOOD + 8), EALIGN),
    (dict(tokens=1 << 30), EUNSUP), (dict(tokens=0), OK),
])
def test_append_refusals(args, want):
    assert append(**args) == want


@pytest.mark.parametrize("kind,dt", [(u.CACHE_F16, u.BF16), (u.CACHE_BF16, u.F16)])
def test_sixteen_bit_kinds_hold_the_activations_type(kind, dt):
    c = cache(kind=kind, ks=None, vs=None)
    assert append(c=c, dt=dt) == EUNSUP
    assert decode(c=c, dt=dt) == EUNSUP


@pytest.mark.parametrize("args,want", [
    (dict(tokens=-1), EINVAL), (dict(cu=None), EINVAL), (dict(k=None), EINVAL), (dict(v=None), EINVAL),
    (dict(dt=u.F32), EINVAL), (dict(kt=100), EALIGN), (dict(v=GOOD + 4), EALIGN), (dict(cu=GOOD + 1), EALIGN),
    (dict(starts=GOOD + 3), EALIGN), (dict(tokens=0), OK), (dict(B=0), OK),
])
def test_read_refusals(args, want):
    assert read(**args) == want


@pytest.mark.parametrize("args,want", [
    (dict(lens=None), EINVAL), (dict(q=None), EINVAL), (dict(out=None), EINVAL), (dict(q_len=0), EINVAL),
    (dict(q_len=17), EINVAL), (dict(qh=3), EINVAL), (dict(qh=1), EINVAL), (dict(scale=0.0), EINVAL),
    (dict(scale=-1.0), EINVAL), (dict(scale=NAN), EINVAL), (dict(scale=INF), EINVAL), (dict(max_len=-1), EINVAL),
    (dict(dt=u.F32), EINVAL), (dict(qt=100), EALIGN), (dict(out=GOOD + 8), EALIGN), (dict(lse=GOOD + 2), EALIGN),
    (dict(lens=GOOD + 2), EALIGN), (dict(width=64, ws=None), EWS), (dict(width=64, size=8), EWS),
    (dict(width=64, ws=GOOD + 8), EALIGN), (dict(B=0), OK), (dict(B=1 << 30, c=cache(heads=64), qh=64), EUNSUP),
])
def test_decode_refusals(args, want):
    assert decode(**args) == want


def prompt(B=2, nq=10, nk=10, cq=GOOD, ck=GOOD, qh=4, kh=2, D=128, q=GOOD, k=GOOD, kt=256, v=GOOD, vt=256, dt=u.F16,
           scale=0.1, out=GOOD, ot=512, lse=None, ws=GOOD, size=1 << 40):
    return u.load().unisvq_attn_prompt(B, nq, nk, cq, ck, qh, kh, D, q, 512, 128, k, kt, 128, v, vt, 128, dt, 1, scale,
                                       out, ot, 128, lse, ws, size, None)


@pytest.mark.parametrize("args,want", [
    (dict(B=-1), EINVAL), (dict(nq=-1), EINVAL), (dict(nk=-1), EINVAL), (dict(nq=1 << 31), EINVAL), (dict(qh=3), EINVAL),
    (dict(kh=0), EINVAL), (dict(dt=u.F32), EINVAL), (dict(scale=0.0), EINVAL), (dict(scale=NAN), EINVAL),
    (dict(D=96), EUNSUP), (dict(cq=None), EINVAL), (dict(ck=None), EINVAL), (dict(q=None), EINVAL),
    (dict(k=None), EINVAL), (dict(v=None), EINVAL), (dict(out=None), EINVAL), (dict(q=GOOD + 2), EALIGN),
    (dict(kt=100), EALIGN), (dict(ot=4), EALIGN), (dict(lse=GOOD + 1), EALIGN), (dict(cq=GOOD + 2), EALIGN),
    (dict(kt=1 << 23), EUNSUP), (dict(vt=-8), EUNSUP), (dict(nq=1 << 30, qh=65532, kh=2), EUNSUP), (dict(B=0), OK),
    (dict(nq=0), OK),
])
def test_prompt_refusals(args, want):
    assert prompt(**args) == want


@pytest.mark.parametrize("call,args", [
    (read, dict(tokens=1 << 28)),  # 2^28 * 2 heads * 8 chunks
    (decode, dict(B=1 << 23, width=1)), (decode, dict(B=1 << 14, width=1 << 23, c=cache(page=16))),
    (prompt, dict(B=1 << 23)),
])
def test_counts_past_a_launch_are_refused(call, args):
    assert call(**args) == EUNSUP


def test_workspace_sizes_of_invalid_shapes_are_zero():
    lib = u.load()
    assert lib.unisvq_attn_decode_workspace_bytes(0, 1, 8, 8, 128, 100) == 0
    assert lib.unisvq_attn_decode_workspace_bytes(1, 0, 8, 8, 128, 100) == 0
    assert lib.unisvq_attn_decode_workspace_bytes(1, 1, 9, 8, 128, 100) == 0
    assert lib.unisvq_attn_decode_workspace_bytes(1, 1, 8, 8, 96, 100) == 0
    assert lib.unisvq_attn_decode_workspace_bytes(1, 1, 8, 8, 128, 100000) > 0
    assert lib.unisvq_attn_prompt_workspace_bytes(0, 1, 1, 8, 8, 128) == 0
    assert lib.unisvq_attn_prompt_workspace_bytes(1, 1, 1, 8, 3, 128) == 0


def test_binding_refuses_host_tensors_and_wrong_shapes():
    torch = pytest.importorskip("torch")
    x = torch.zeros((3, 2, 128), dtype=torch.float16)
    pos = torch.zeros(3, dtype=torch.int32)
    t = torch.zeros((8, 2, 64))
    with pytest.raises(ValueError):
        u.rope(x, pos, t)  # host tensors
    with pytest.raises(ValueError):
        u.rope(x.reshape(3, 256), pos, t)
    pools = torch.zeros((4, 2, 64, 128), dtype=torch.int8)
    with pytest.raises(ValueError):
        u.cache_read((pools, pools, None, None), pos.reshape(1, 3), None, pos, 3)
    with pytest.raises(TypeError):
        u.cache_read((pools.float(), pools.float(), None, None), pos.reshape(1, 3), None, pos, 3)


def test_cache_struct_matches_the_header():
    assert ctypes.sizeof(u.Cache) == 72
