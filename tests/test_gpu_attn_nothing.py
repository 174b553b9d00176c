"""Calls over which there is nothing to see at all: no keys in any sequence, no columns in the page table, empty batches."""
import pytest

from test_gpu_attn_prompt import DEV, ints, u  # noqa: F401  (u is a fixture)

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("D", [64, 128])
def test_prompts_without_keys(u, causal, D):  # noqa: F811
    q = torch.randn((7, 4, D), device=DEV).half()
    none = torch.empty((0, 2, D), dtype=torch.float16, device=DEV)
    lse = torch.zeros((7, 4), device=DEV)
    out = u.attn_prompt(q, none, none, ints([0, 5, 7]), ints([0, 0, 0]), causal=causal, lse=lse)
    assert not out.any() and torch.isneginf(lse).all()
    assert u.attn_prompt(q[:0], none, none, ints([0, 0, 0]), ints([0, 0, 0]), causal=causal).shape == (0, 4, D)


@pytest.mark.parametrize("kind", ["i8", "i4", "f16"])
@pytest.mark.parametrize("q_len", [1, 3])
def test_page_tables_without_columns(u, kind, q_len):  # noqa: F811
    cache = u.new_cache(1, 2, 16, 128, kind)
    q = torch.randn((3, q_len, 8, 128), device=DEV).half()
    lse = torch.zeros((3, q_len, 8), device=DEV)
    table = torch.empty((3, 0), dtype=torch.int32, device=DEV)
    out = u.attn_decode(q, cache, table, ints([5, 0, 2 ** 31 - 1]), lse=lse)
    assert not out.any() and torch.isneginf(lse).all()
    k = torch.randn((3, 2, 128), device=DEV).half()
    u.cache_append(cache, table, None, ints([0, 1, 2]), k, k)
    assert not any(t.any() for t in cache if t is not None)
    got, _ = u.cache_read(cache, table, None, ints([0, 1, 1, 2]), 2, out_dtype=torch.float16)
    assert torch.isnan(got).all()


@pytest.mark.parametrize("kind", ["i8", "f16"])
def test_empty_batches(u, kind):  # noqa: F811
    cache = u.new_cache(1, 2, 16, 64, kind)
    table = torch.empty((0, 4), dtype=torch.int32, device=DEV)
    q = torch.empty((0, 8, 64), dtype=torch.float16, device=DEV)
    assert u.attn_decode(q, cache, table, ints([])).shape == (0, 8, 64)
    k = torch.empty((0, 2, 64), dtype=torch.float16, device=DEV)
    assert u.cache_append(cache, table, ints([]), ints([]), k, k, q=q).shape == (0, 8, 64)
    assert u.cache_read(cache, table, None, ints([0]), 0, out_dtype=torch.float16)[0].shape == (0, 2, 64)
