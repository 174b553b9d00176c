"""Attention over prompts at the grids that large calls have: more workgroups than CUs, paired by their work; more than
the GPU holds at once; either with split keys; key heads spread over the dies.  Against 64 bits, a few heads each."""
import numpy as np
import pytest

import attn_ref as ref
from test_gpu_attn_prompt import DEV, cum, ints, make, u  # noqa: F401  (u is a fixture)

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


def grid(u, nq, nk, HQ, H, D):
    """Workgroups of the call and parts of a tile's keys (as the workspace tells)."""
    need = u.attn_prompt_workspace_bytes(len(nq), sum(nq), sum(nk), HQ, H, D)
    splits = max(1, need // (sum(nq) * HQ * (D + 2) * 4))
    return (sum(nq) * (HQ // H) + 127 * len(nq)) // 128 * H * splits, splits


def check_heads(u, nq, nk, HQ, H, D, dtype, causal, heads, seed):
    q, k, v = make(nq, nk, HQ, H, D, dtype, seed)
    cq, ck = cum(nq), cum(nk)
    out = torch.full(q.shape, 123.0, dtype=q.dtype, device=DEV)
    lse = torch.full(q.shape[:2], 123.0, device=DEV)
    u.attn_prompt(q.to(DEV), k.to(DEV), v.to(DEV), ints(cq), ints(ck), causal=causal, out=out, lse=lse)
    assert not (lse == 123).any()
    out, lse = out.double().cpu().numpy(), lse.double().cpu().numpy()
    for b in range(len(nq)):
        last = np.arange(nq[b]) + nk[b] - nq[b] if causal else np.full(nq[b], nk[b])
        rows, keys = slice(cq[b], cq[b + 1]), slice(ck[b], ck[b + 1])
        for h in heads:
            at = h * H // HQ
            kb, vb = (x[keys, at:at + 1].double().numpy() for x in (k, v))
            r = ref.attention(q[rows, h:h + 1].double().numpy(), kb, vb, last, D ** -0.5)
            ref.check(out[rows, h:h + 1], lse[rows, h:h + 1], r, max(1, nk[b]), dtype, dtype, np.abs(vb).max() if vb.size else 0.0)


RAGGED = [700, 1, 0, 900, 333, 128, 129, 0, 511, 64, 2, 800]


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("nq,nk,HQ,H,D,heads", [
    ([1300], [1300], 32, 32, 128, [0, 5, 30]),
    (RAGGED, RAGGED, 8, 8, 64, [0, 3, 7]),
    (RAGGED, [n + 100 for n in RAGGED], 8, 8, 128, [1, 6]),
])
def test_workgroups_paired_by_their_work(u, dtype, causal, nq, nk, HQ, H, D, heads):  # noqa: F811
    blocks, splits = grid(u, nq, nk, HQ, H, D)
    assert splits == 1 and 256 < blocks <= 512 and 256 % H == 0
    check_heads(u, nq, nk, HQ, H, D, dtype, causal, heads, 1)


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("nq,HQ,H,D,heads", [
    ([2500], 32, 32, 128, [0, 17]), ([2000, 1, 1500], 32, 4, 64, [0, 9]), ([1100, 0, 900, 1], 40, 40, 128, [3, 39]),
])
def test_more_workgroups_than_the_gpu_holds(u, dtype, nq, HQ, H, D, heads):  # noqa: F811
    blocks, splits = grid(u, nq, nq, HQ, H, D)
    assert splits == 1 and blocks > 512
    check_heads(u, nq, nq, HQ, H, D, dtype, True, heads, 2)


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("nq,nk,HQ,H,D,heads", [
    ([150, 50], [3500, 500], 64, 8, 128, [0, 13, 63]), ([128, 1, 127], [2500, 1500, 2000], 16, 16, 128, [0, 9]),
    ([200, 100], [2000, 1000], 32, 32, 64, [2, 31]),
])
def test_paired_parts_of_keys(u, causal, nq, nk, HQ, H, D, heads):  # noqa: F811
    blocks, splits = grid(u, nq, nk, HQ, H, D)
    assert splits > 1 and 256 < blocks <= 512 and 256 % (H * splits) == 0
    check_heads(u, nq, nk, HQ, H, D, "bf16", causal, heads, 3)
