"""The example of a served attention block: projections, rotary positions, cache and attention together."""
import importlib.util
import os

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

PATH = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "attention_block.py")


@pytest.fixture(scope="module")
def example():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    spec = importlib.util.spec_from_file_location("attention_block", PATH)
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


# the chain rounds to fp16 about ten times (2^-11 each, some amplified by the scores); 8-bit codes are off by up to
# 1/254 of a head's largest value (three to four times its rms), 4-bit ones by 1/14
@pytest.mark.parametrize("kind,bound", [("f16", 0.01), ("i8", 0.03), ("i4", 0.35)])
@pytest.mark.parametrize("heads,kv_heads", [(8, 2), (16, 16)])
def test_generation_matches_the_dense_block(example, kind, bound, heads, kv_heads):
    assert example.run(kind, 1024, heads, kv_heads) <= bound


def test_prompt_in_chunks_is_the_prompt_at_once(example):
    """Chunks of a prompt after what is cached of it give what one pass gives, up to the cache's rounding (f16: none)."""
    u = example.u
    made = [example.random_weights(n, 512, seed)[0] for seed, n in enumerate((512, 128, 128, 512))]
    x = torch.randn((100, 512), device="cuda").half()
    outs = []
    for parts in ((100,), (37, 1, 62)):
        block = example.AttentionBlock(512, 4, 1, made, "f16", 1, 128)
        outs.append(torch.cat([block.prefill(p, [p.shape[0]]) for p in x.split(parts)]))
    err = (outs[0].float() - outs[1].float()).norm() / outs[0].float().norm()
    assert err <= 4e-3  # other kernels for other token counts: a few fp16 roundings apart


def test_new_memory_is_the_streams_own():
    """What a call makes for another stream must not be memory that the current stream may still be using."""
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2606_10520_amd.unisvq as u
    x = torch.randn((1000, 8, 64), device="cuda").half()
    pos = torch.arange(1000, dtype=torch.int32, device="cuda")
    cu = torch.tensor([0, 1000], dtype=torch.int32, device="cuda")
    s, table = torch.cuda.Stream(), u.rope_table(1000, 64)
    torch.cuda.synchronize()
    for call in (lambda: u.rope(x, pos, table, stream=s), lambda: u.attn_prompt(x, x, x, cu, cu, stream=s)):
        freed = torch.empty_like(x)
        at = freed.data_ptr()
        del freed
        assert torch.empty_like(x).data_ptr() == at  # the current stream would get it again
        out = call()
        assert out.data_ptr() != at
        s.synchronize()
