"""Refusals of the norm, gating and 4-bit entry points (every call fails validation or has nothing to do, so no kernel is
launched and the addresses are never read), and the device and stream that a call of the binding runs on."""
import ctypes
import os
import types

import pytest

import paper_2606_10520_amd.unisvq as u

torch = pytest.importorskip("torch")
built = pytest.mark.skipif(not os.path.exists(u.LIB_PATH), reason="libunisvq.so not built")

OK, EINVAL, ESHAPE, EUNSUP, EALIGN, EWS = 0, -1, -2, -3, -4, -6
GOOD = 0x10000
NAN, INF = float("nan"), float("inf")


def norm(tokens=4, n=256, x=GOOD, xs=256, xt=u.F16, w=GOOD, wt=u.F16, off=0.0, eps=1e-5, r=GOOD, rs=256, h=GOOD, hs=256,
         rt=u.F16, y=GOOD, ys=256, yt=u.F16, s=GOOD):
    return u.load().unisvq_rmsnorm(tokens, n, x, xs, xt, w, wt, off, eps, r, rs, h, hs, rt, y, ys, yt, s, None)


@built
@pytest.mark.parametrize("args,want", [
    (dict(tokens=-1), EINVAL), (dict(tokens=1 << 31), EINVAL), (dict(n=0), EINVAL), (dict(xt=u.F32), EINVAL),
    (dict(xt=9), EINVAL), (dict(x=None), EINVAL), (dict(w=None), EINVAL), (dict(y=None), EINVAL), (dict(eps=0.0), EINVAL),
    (dict(eps=-1e-5), EINVAL), (dict(eps=NAN), EINVAL), (dict(eps=INF), EINVAL), (dict(off=NAN), EINVAL),
    (dict(r=None), EINVAL), (dict(h=None), EINVAL), (dict(yt=u.I8, s=None), EINVAL), (dict(yt=7), EINVAL),
    (dict(wt=7), EINVAL), (dict(rt=7), EINVAL), (dict(wt=u.I8), EINVAL), (dict(rt=u.I8), EINVAL),
    (dict(wt=u.BF16), EUNSUP), (dict(rt=u.BF16), EUNSUP), (dict(yt=u.BF16), EUNSUP), (dict(n=260), EUNSUP),
    (dict(n=65544), EUNSUP), (dict(x=GOOD + 2), EALIGN), (dict(xs=257), EALIGN), (dict(w=GOOD + 8), EALIGN),
    (dict(r=GOOD + 8), EALIGN), (dict(rs=4), EALIGN), (dict(h=GOOD + 8), EALIGN), (dict(hs=258), EALIGN),
    (dict(y=GOOD + 8), EALIGN), (dict(ys=1), EALIGN), (dict(yt=u.I8, s=GOOD + 2), EALIGN), (dict(tokens=0), OK),
    (dict(tokens=0, x=None, y=None, r=None, h=None), OK),
])
def test_norm_refusals(args, want):
    assert norm(**args) == want


def gated(tokens=4, n=256, g=GOOD, gs=256, v=GOOD, vs=256, xt=u.F16, act=0, y=GOOD, ys=256, yt=u.F16, s=GOOD):
    return u.load().unisvq_gated(tokens, n, g, gs, v, vs, xt, act, y, ys, yt, s, None)


@built
@pytest.mark.parametrize("args,want", [
    (dict(tokens=-1), EINVAL), (dict(n=0), EINVAL), (dict(xt=u.F32), EINVAL), (dict(xt=u.I8), EINVAL), (dict(g=None), EINVAL),
    (dict(v=None), EINVAL), (dict(y=None), EINVAL), (dict(act=2), EINVAL), (dict(act=-1), EINVAL),
    (dict(yt=u.I8, s=None), EINVAL), (dict(yt=u.BF16), EUNSUP), (dict(n=12), EUNSUP), (dict(yt=u.I8, n=65544, ys=65544), EUNSUP),
    (dict(tokens=1 << 30, n=1 << 10), EUNSUP), (dict(n=1 << 32), EUNSUP), (dict(g=GOOD + 4), EALIGN), (dict(vs=4), EALIGN),
    (dict(y=GOOD + 2), EALIGN), (dict(ys=9), EALIGN), (dict(tokens=0), OK),
])
def test_gated_refusals(args, want):
    assert gated(**args) == want


@built
@pytest.mark.parametrize("args", [
    dict(), dict(r=None, h=None, ys=512), dict(r=None, h=None, yt=u.F32), dict(r=None, h=None, yt=u.I8), dict(y=2 * GOOD, hs=512),
    dict(y=2 * GOOD, rt=u.F32), dict(h=2 * GOOD, rt=u.F32), dict(h=2 * GOOD, rs=512), dict(y=2 * GOOD, ys=128),
    dict(y=2 * GOOD, ys=0), dict(y=2 * GOOD, ys=-248), dict(y=2 * GOOD, x=3 * GOOD, r=4 * GOOD, hs=0), dict(eps=1e-39)])
def test_norm_refuses_outputs_that_overlap(args):
    """Outputs on one another's or their own other rows, or on an input that is not the same rows of the same type; and an
    eps below the normal numbers."""
    assert norm(**args) == EINVAL


@built
@pytest.mark.parametrize("args", [dict(yt=u.F32), dict(yt=u.I8), dict(ys=512), dict(g=2 * GOOD, vs=512), dict(y=2 * GOOD, ys=248)])
def test_gated_refuses_outputs_that_overlap(args):
    assert gated(**args) == EINVAL


def gemm(N=256, K=256, p=GOOD, M=4, x=GOOD, xt=u.F16, xs=None, y=2 * GOOD, yt=u.F16, ws=GOOD, size=1 << 40):
    return u.load().unisvq_fourbit_gemm(N, K, p, M, x, xt, xs, y, yt, ws, size, None)


BAD = [(dict(p=None), EINVAL), (dict(x=None), EINVAL), (dict(y=None), EINVAL), (dict(M=0), EINVAL), (dict(M=1 << 31), EINVAL),
       (dict(xt=u.F32), EINVAL), (dict(xt=9), EINVAL), (dict(yt=u.I8), EINVAL), (dict(yt=9), EINVAL),
       (dict(xt=u.I8), EINVAL), (dict(xs=GOOD), EINVAL), (dict(N=8), ESHAPE), (dict(N=24), ESHAPE), (dict(K=64), ESHAPE),
       (dict(K=192), ESHAPE), (dict(N=0), ESHAPE), (dict(K=(1 << 20) + 128), EUNSUP), (dict(p=GOOD + 8), EALIGN),
       (dict(x=GOOD + 8), EALIGN), (dict(y=GOOD + 1), EALIGN), (dict(y=GOOD + 2, yt=u.F32), EALIGN),
       (dict(xt=u.I8, xs=GOOD + 2), EALIGN)]


@built
@pytest.mark.parametrize("args,want", BAD)
def test_fourbit_gemm_refusals(args, want):
    assert gemm(**args) == want


@built
@pytest.mark.parametrize("args,want", BAD)
def test_fourbit_batched_refusals(args, want):
    """The last of a batch is looked at as the first is."""
    a = dict(N=256, K=256, p=GOOD, M=4, x=GOOD, xt=u.F16, xs=None, y=2 * GOOD, yt=u.F16)
    a.update(args)
    good_scales = GOOD if a["xt"] == u.I8 else None
    arr = (u.FourbitProblem * 2)((256, 256, GOOD, GOOD, good_scales, 3 * GOOD), (a["N"], a["K"], a["p"], a["x"], a["xs"], a["y"]))
    assert u.load().unisvq_fourbit_gemm_batched(arr, 2, a["M"], a["xt"], a["yt"], GOOD, 1 << 40, None) == want


@built
@pytest.mark.parametrize("ys", [(2 * GOOD, 2 * GOOD), (GOOD, 2 * GOOD), (2 * GOOD, 5 * GOOD), (7 * GOOD, 2 * GOOD)])
def test_fourbit_outputs_that_overlap(ys):
    """Two problems' outputs, or an output and some problem's activations or weights, in one place."""
    arr = (u.FourbitProblem * 2)((256, 256, 4 * GOOD, GOOD, None, ys[0]), (256, 256, 5 * GOOD, 7 * GOOD, None, ys[1]))
    assert u.load().unisvq_fourbit_gemm_batched(arr, 2, 4, u.F16, u.F16, GOOD, 1 << 40, None) == EINVAL


@built
def test_fourbit_counts_sizes_and_workspaces():
    lib = u.load()
    arr = (u.FourbitProblem * 1)((256, 256, GOOD, GOOD, None, GOOD))
    for count in (0, -1, 9):
        assert lib.unisvq_fourbit_gemm_batched(arr, count, 4, u.F16, u.F16, GOOD, 1 << 40, None) == EINVAL
        assert lib.unisvq_fourbit_gemm_batched_workspace_bytes(arr, count, 4, u.F16) == 0
    assert lib.unisvq_fourbit_gemm_batched(None, 1, 4, u.F16, u.F16, GOOD, 1 << 40, None) == EINVAL
    assert u.fourbit_bytes(16, 128) == 1024 + 128 and u.fourbit_bytes(4096, 4096) == 4096 * 2048 + 4096 * 64
    for N, K in ((0, 128), (16, 0), (8, 128), (16, 64), (16, (1 << 20) + 128), (-16, 128)):
        assert u.fourbit_bytes(N, K) == 0 and lib.unisvq_fourbit_gemm_workspace_bytes(N, K, 4, u.F16) == 0
    for N, K, M in ((4096, 4096, 1), (16, 1 << 20, 100), (1024, 8192, 100), (8192, 28672, 64), (528, 4096, 2500)):
        for t in (u.F16, u.BF16, u.I8):
            need = lib.unisvq_fourbit_gemm_workspace_bytes(N, K, M, t)
            assert need < 1 << 31 and need % 16 == 0
            if need:
                scales = GOOD if t == u.I8 else None
                assert gemm(N, K, M=M, xt=t, xs=scales, size=need - 1) == EWS
                assert gemm(N, K, M=M, xt=t, xs=scales, ws=None) == EWS
                assert gemm(N, K, M=M, xt=t, xs=scales, ws=GOOD + 8) == EALIGN


@built
def test_fourbit_packing_refusals():
    lib = u.load()
    good = dict(N=32, K=256, a=GOOD, b=GOOD, p=GOOD)
    cases = [(dict(a=None), EINVAL), (dict(p=None), EINVAL), (dict(N=24), ESHAPE), (dict(K=100), ESHAPE), (dict(p=GOOD + 4), EALIGN),
             (dict(K=(1 << 20) + 128), EUNSUP)]
    for args, want in cases + [(dict(b=None), EINVAL), (dict(b=GOOD + 1), EALIGN)]:
        c = {**good, **args}
        assert lib.unisvq_fourbit_pack(c["N"], c["K"], c["a"], c["b"], c["p"], None, None) == want
        assert lib.unisvq_fourbit_unpack(c["N"], c["K"], c["p"], c["a"], c["b"], None) == want
    for args, want in cases + [(dict(a=GOOD + 8), EALIGN)]:
        c = {**good, **args}
        assert lib.unisvq_fourbit_quantize(c["N"], c["K"], c["a"], u.F32, c["p"], None) == want
    assert lib.unisvq_fourbit_quantize(32, 256, GOOD, u.I8, GOOD, None) == EINVAL


# ---- the binding: devices, streams and its own refusals, with stand-ins for device tensors and the library ----

class On:
    """A host tensor that says it is on device `index`."""

    def __init__(self, t, index):
        self.t, self.index, self.is_cuda = t, index, True
        self.device = torch.device("cuda", index)

    def __getattr__(self, name):
        return getattr(self.t, name)

    def get_device(self):
        return self.index

    def new_empty(self, shape, dtype):
        return On(torch.empty(shape, dtype=dtype), self.index)


@pytest.fixture
def calls(monkeypatch):
    """The calls that reach the library, as (name, current device, stream); device 0 is current."""
    made, state = [], types.SimpleNamespace(current=0)

    class Library:
        def __getattr__(self, name):
            if name == "unisvq_fourbit_bytes":
                return lambda N, K: N * K // 2 + N * 8 * -(-K // 512)
            if name.endswith("_bytes"):
                return lambda *a: 64
            return lambda *a: made.append((name, state.current, a[-1])) or 0

    class Device:
        def __init__(self, index):
            self.index = index

        def __enter__(self):
            self.was, state.current = state.current, self.index

        def __exit__(self, *_):
            state.current = self.was

    monkeypatch.setattr(u, "load", lambda: Library())
    monkeypatch.setattr(u, "_current", (lambda: state.current, lambda index: 1000 + index), raising=False)
    monkeypatch.setattr(u, "_new", lambda shape, dtype, device, stream: On(torch.empty(shape, dtype=dtype), torch.device(device).index))
    monkeypatch.setattr(torch.cuda, "device", Device)
    monkeypatch.setattr(torch, "empty_like", lambda t, dtype: t.new_empty(t.shape, dtype))
    u._fourbit_workspace.cache_clear(), u._fourbit_size.cache_clear()
    yield made
    u._fourbit_workspace.cache_clear(), u._fourbit_size.cache_clear()


def arguments(op, at):
    """A call of op, its tensors all on device at[name] or 1."""
    def t(name, *shape, dtype=torch.float16):
        return On(torch.zeros(shape, dtype=dtype), at.get(name, 1))
    ws = t("workspace", 64, dtype=torch.uint8)
    packed = t("packed", 32 * 128 + 32 * 8, dtype=torch.uint8)
    if op == "norm":
        return u.rmsnorm, (t("x", 3, 64), t("weight", 64)), dict(residual=t("residual", 3, 64), residual_out=t("h", 3, 64), out=t("out", 3, 64))
    if op == "norm_i8":
        return u.rmsnorm, (t("x", 3, 64), t("weight", 64)), dict(out=(t("out", 3, 64, dtype=torch.int8), t("scales", 3, dtype=torch.float32)))
    if op == "gated":
        return u.gated, (t("gate", 3, 64), t("up", 3, 64)), dict(out=t("out", 3, 64))
    if op == "pack":
        return u.fourbit_pack, (t("codes", 32, 256, dtype=torch.uint8), t("scales", 32, 2)), dict(out=packed, bad_codes=t("bad", 1, dtype=torch.int32))
    if op == "unpack":
        return u.fourbit_unpack, (packed, 32, 256), {}
    if op == "quantize":
        return u.fourbit_quantize, (t("W", 32, 256),), dict(out=packed)
    if op == "gemm_i8":
        x = t("x", 3, 256, dtype=torch.int8), t("scales", 3, dtype=torch.float32)
        return u.fourbit_gemm, (packed, 32, 256, x), dict(out=t("out", 3, 32), workspace=ws)
    return u.fourbit_gemm, (packed, 32, 256, t("x", 3, 256)), dict(out=t("out", 3, 32), workspace=ws)


USED = {"norm": ["x", "weight", "residual", "h", "out"], "norm_i8": ["x", "out", "scales"], "gated": ["gate", "up", "out"],
        "pack": ["codes", "scales", "packed", "bad"], "unpack": [], "quantize": ["W", "packed"],
        "gemm": ["packed", "x", "out", "workspace"], "gemm_i8": ["x", "scales", "out"]}


@pytest.mark.parametrize("op", USED)
def test_a_call_runs_on_its_tensors_device(calls, op):
    f, args, more = arguments(op, {})
    f(*args, **more)
    assert [c[1:] for c in calls] == [(1, 1001)]


@pytest.mark.parametrize("op", USED)
def test_a_call_without_outputs_makes_them(calls, op):
    f, args, _ = arguments(op, {})
    out = f(*args)
    assert [c[1:] for c in calls] == [(1, 1001)]
    assert (out[0] if isinstance(out, tuple) else out).get_device() == 1


@pytest.mark.parametrize("op,name", [(op, name) for op in USED for name in USED[op]])
def test_tensors_of_two_devices_are_refused(calls, op, name):
    f, args, more = arguments(op, {name: 2})
    with pytest.raises(ValueError):
        f(*args, **more)
    assert calls == []


@pytest.mark.parametrize("op", USED)
def test_a_stream_of_another_device_is_refused(calls, op):
    f, args, more = arguments(op, {})
    with pytest.raises(ValueError):
        f(*args, **more, stream=types.SimpleNamespace(device=torch.device("cuda", 0), cuda_stream=7))
    assert calls == []
    f(*args, **more, stream=types.SimpleNamespace(device=torch.device("cuda", 1), cuda_stream=8))
    assert [c[1:] for c in calls] == [(1, 8)]


def test_the_binding_refuses_what_does_not_fit(calls):
    def t(*shape, dtype=torch.float16):
        return On(torch.zeros(shape, dtype=dtype), 1)
    x, w, packed = t(3, 64), t(64), t(32 * 128 + 32 * 8, dtype=torch.uint8)
    x8 = t(3, 256, dtype=torch.int8), t(3, dtype=torch.float32)
    for f in (lambda: u.rmsnorm(t(3, 64, dtype=torch.float32), w), lambda: u.rmsnorm(x, t(63)), lambda: u.rmsnorm(x, w, residual_out=x),
              lambda: u.rmsnorm(x, t(64, dtype=torch.bfloat16)), lambda: u.rmsnorm(x, w, residual=t(2, 64)),
              lambda: u.rmsnorm(x, w, residual=t(3, 64, dtype=torch.bfloat16)),
              lambda: u.rmsnorm(x, w, residual=x, residual_out=t(3, 64, dtype=torch.float32)), lambda: u.rmsnorm(x, w, out=t(3, 32)),
              lambda: u.rmsnorm(x, w, out=t(3, 64, dtype=torch.int8)), lambda: u.rmsnorm(x, w, out=(x, t(3, dtype=torch.float32))),
              lambda: u.rmsnorm(x, w, out=t(3, 64, dtype=torch.float64)), lambda: u.rmsnorm(x, w, out=x, out_dtype=torch.float32),
              lambda: u.rmsnorm(x, w, out=(t(3, 64, dtype=torch.int8), t(2, dtype=torch.float32))),
              lambda: u.rmsnorm(On(torch.zeros(64, 3).half().T, 1), w), lambda: u.rmsnorm(t(64), w),
              lambda: u.gated(x, t(3, 32)), lambda: u.gated(x, t(3, 64, dtype=torch.bfloat16)), lambda: u.gated(x, x, "relu"),
              lambda: u.fourbit_gemm(packed, 32, 256, t(3, 128)), lambda: u.fourbit_gemm(packed, 32, 256, t(3, 256, dtype=torch.float32)),
              lambda: u.fourbit_gemm(packed, 32, 256, x8[0]), lambda: u.fourbit_gemm(packed, 32, 256, (t(3, 256), x8[1])),
              lambda: u.fourbit_gemm(packed, 32, 256, (x8[0], t(2, dtype=torch.float32))), lambda: u.fourbit_gemm(packed, 16, 256, t(3, 256)),
              lambda: u.fourbit_gemm(packed, 32, 256, t(3, 256), out=t(3, 16)), lambda: u.fourbit_gemm(packed, 32, 256, t(0, 256)),
              lambda: u.fourbit_gemm(packed, 32, 256, t(3, 256), out=t(3, 32, dtype=torch.int8)),
              lambda: u.fourbit_gemm(packed, 32, 256, t(3, 256), out=t(3, 32), out_dtype=torch.float32),
              lambda: u.fourbit_gemm(packed, 32, 256, t(3, 256), workspace=t(8, dtype=torch.uint8)),
              lambda: u.fourbit_gemm(packed, 32, 256, On(torch.zeros(3, 512).half()[:, ::2], 1)),
              lambda: u.fourbit_gemm_batched([]), lambda: u.fourbit_gemm_batched([(packed, 32, 256, t(3, 256), None)] * 9),
              lambda: u.fourbit_gemm_batched([(packed, 32, 256, t(3, 256), None), (packed, 32, 256, t(2, 256), None)]),
              lambda: u.fourbit_gemm_batched([(packed, 32, 256, t(3, 256), None), (packed, 32, 256, x8, None)]),
              lambda: u.fourbit_gemm_batched([(packed, 32, 256, t(3, 256), t(3, 32)), (packed, 32, 256, t(3, 256), t(3, 32, dtype=torch.float32))]),
              lambda: u.fourbit_pack(t(32, 256), t(32, 2)), lambda: u.fourbit_pack(t(32, 256, dtype=torch.uint8), t(32, 1)),
              lambda: u.fourbit_quantize(t(32, 256, dtype=torch.float64)), lambda: u.fourbit_unpack(t(7, dtype=torch.uint8), 32, 256)):
        with pytest.raises((ValueError, TypeError)):
            f()
    assert calls == []
