"""Which device a call of the attention block runs on, with stand-ins for device tensors and for the library: nothing is
launched."""
import types

import pytest

torch = pytest.importorskip("torch")
import paper_2606_10520_amd.unisvq as u  # noqa: E402


class On:
    """A host tensor that says it is on device `index`."""

    def __init__(self, t, index):
        self.t, self.index, self.is_cuda = t, index, True
        self.device = torch.device("cuda", index)

    def __getattr__(self, name):
        return getattr(self.t, name)

    def get_device(self):
        return self.index

    def view(self, *shape):
        return On(self.t.view(*shape), self.index)


@pytest.fixture
def calls(monkeypatch):
    """The calls that reach the library, as (name, current device, stream); device 0 is current."""
    made, state = [], types.SimpleNamespace(current=0)

    class Library:
        def __getattr__(self, name):
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
    u._workspace_size.cache_clear()
    yield made
    u._workspace_size.cache_clear()
    assert state.current == 0


def arguments(op, at):
    """A call of op, its tensors all on device at[name] or 1."""
    def t(name, *shape, dtype=torch.float16):
        return On(torch.zeros(shape, dtype=dtype), at.get(name, 1))
    rows = {n: t(n, 3, h, 64) for n, h in (("q", 4), ("k", 2), ("v", 2), ("out", 4))}
    words = lambda name, n: t(name, n, dtype=torch.int32)
    cache = (t("pool_k", 5, 2, 16, 64, dtype=torch.int8), t("pool_v", 5, 2, 16, 64, dtype=torch.int8),
             t("scales_k", 5, 2, 16, dtype=torch.float32), t("scales_v", 5, 2, 16, dtype=torch.float32))
    pages, table = t("pages", 3, 2, dtype=torch.int32), t("table", 9, 2, 32, dtype=torch.float32)
    lse, ws = t("lse", 12, dtype=torch.float32), t("workspace", 64, dtype=torch.uint8)
    if op == "rope":
        return u.rope, (rows["q"], words("positions", 3), table), dict(out=rows["out"])
    if op == "append":
        return u.cache_append, (cache, pages, words("seqs", 3), words("positions", 3), rows["k"], rows["v"]), \
            dict(q=rows["q"], rope_table=table, q_out=rows["out"])
    if op == "read":
        return u.cache_read, (cache, pages, words("starts", 3), words("cu", 4), 3), dict(out=(rows["k"], rows["v"]))
    if op == "decode":
        return u.attn_decode, (rows["q"], cache, pages, words("lens", 3)), dict(out=rows["out"], lse=lse, workspace=ws)
    return u.attn_prompt, (rows["q"], rows["k"], rows["v"], words("cu_q", 2), words("cu_k", 2)), \
        dict(out=rows["out"], lse=lse, workspace=ws)


CACHE = ["pool_k", "pool_v", "scales_k", "scales_v", "pages"]
USED = {"rope": ["q", "positions", "table", "out"],
        "append": CACHE + ["seqs", "positions", "k", "v", "q", "table", "out"],
        "read": CACHE + ["starts", "cu", "k", "v"],
        "decode": CACHE + ["q", "lens", "out", "lse", "workspace"],
        "prompt": ["q", "k", "v", "cu_q", "cu_k", "out", "lse", "workspace"]}


@pytest.mark.parametrize("op", USED)
def test_a_call_runs_on_its_tensors_device(calls, op):
    f, args, more = arguments(op, {})
    f(*args, **more)
    assert [c[1:] for c in calls] == [(1, 1001)]


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


def test_a_new_table_is_made_on_its_device(calls):
    assert u.rope_table(9, 64, device="cuda:1").get_device() == 1
    assert [c[1:] for c in calls] == [(1, 1001)]


def test_a_table_in_host_memory_is_refused(calls):
    with pytest.MonkeyPatch.context() as m:
        m.setattr(u, "_new", lambda shape, dtype, device, stream: torch.empty(shape, dtype=dtype))
        with pytest.raises(ValueError):
            u.rope_table(9, 64, device="cpu")
    assert calls == []
