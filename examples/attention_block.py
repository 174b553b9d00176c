"""The attention half of a decoder layer, served: 2-bit quantised projections around rotary positions, a paged cache and
attention.  A batch of prompts of different lengths goes through in one pass, then tokens are generated one at a time.

    python examples/attention_block.py [--kind i8] [--hidden 1024] [--heads 8] [--kv-heads 2]

prints the time of both and how far the last step is from the same step computed densely in fp32.
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2606_10520_amd.unisvq as u  # noqa: E402


class AttentionBlock:
    """x -> x W_q, x W_k, x W_v -> rotary positions -> cache -> attention -> W_o, with packed weights (format v1)."""

    def __init__(self, hidden, heads, kv_heads, weights, kind, sequences, max_len, page_tokens=64, dtype=torch.float16):
        self.hidden, self.heads, self.kv_heads, self.D = hidden, heads, kv_heads, hidden // heads
        self.wq, self.wk, self.wv, self.wo = weights
        width = -(-max_len // page_tokens)
        self.cache = u.new_cache(sequences * width, kv_heads, page_tokens, self.D, kind)
        # any assignment of pages will do; a server hands them out as sequences grow
        self.pages = torch.randperm(sequences * width, device="cuda").to(torch.int32).view(sequences, width)
        self.lens = torch.zeros(sequences, dtype=torch.int32, device="cuda")
        self.rope = u.rope_table(max_len, self.D)

    def _project(self, x):
        kv = self.kv_heads * self.D
        problems = [(self.wq, self.hidden, self.hidden, x, None), (self.wk, kv, self.hidden, x, None),
                    (self.wv, kv, self.hidden, x, None)]
        q, k, v = u.gemm_batched(problems)
        return (t.view(x.shape[0], -1, self.D) for t in (q, k, v))

    def _out(self, o):
        return u.gemm(self.wo, self.hidden, self.hidden, o.reshape(o.shape[0], self.hidden))

    def prefill(self, x, counts):
        """x [tokens][hidden]: counts[b] new tokens of every sequence b, after what its cache holds."""
        n = torch.tensor(counts, dtype=torch.int32, device=x.device)
        zero = torch.zeros(1, dtype=torch.int32, device=x.device)
        seqs = torch.repeat_interleave(torch.arange(len(counts), device=x.device), n.long()).to(torch.int32)
        cu_q = torch.cat([zero, n.cumsum(0).to(torch.int32)])
        positions = (torch.arange(x.shape[0], device=x.device) - cu_q[seqs.long()] + self.lens[seqs.long()]).to(torch.int32)
        q, k, v = self._project(x)
        q = u.cache_append(self.cache, self.pages, seqs, positions, k, v, q=q, rope_table=self.rope, q_out=q)
        self.lens += n
        cu_k = torch.cat([zero, self.lens.cumsum(0).to(torch.int32)])
        k, v = u.cache_read(self.cache, self.pages, None, cu_k, int(cu_k[-1]), out_dtype=x.dtype)
        return self._out(u.attn_prompt(q, k, v, cu_q, cu_k))

    def step(self, x):
        """x [sequences][hidden]: the next token of every sequence."""
        q, k, v = self._project(x)
        q = u.cache_append(self.cache, self.pages, None, self.lens, k, v, q=q, rope_table=self.rope, q_out=q)
        self.lens += 1
        return self._out(u.attn_decode(q, self.cache, self.pages, self.lens))


def random_weights(N, K, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    codes = torch.randint(0, 4, (N, K), generator=g, device="cuda", dtype=torch.uint8)
    a = (torch.randn((N, K // u.GROUP, 4, 4), generator=g, device="cuda") * 0.02).half()
    b = (torch.randn((N, K // u.GROUP, 4), generator=g, device="cuda") * 0.01).half()
    dense = torch.einsum("ngab,ngvb->ngva", a.float(), codes.view(N, K // u.GROUP, 32, 4).float()) + b.float()[:, :, None]
    return u.pack(codes, a, b), dense.reshape(N, K)


def dense_last(x, dense, heads, kv_heads):
    """The block's output for the last token of one sequence x [tokens][hidden], in fp32."""
    wq, wk, wv, wo = dense
    n, D = x.shape[0], wq.shape[0] // heads
    q, k, v = ((x @ w.T).view(n, -1, D) for w in (wq, wk, wv))
    freq = 10000.0 ** (-torch.arange(0, D, 2, dtype=torch.float64, device=x.device) / D)
    angle = torch.arange(n, dtype=torch.float64, device=x.device)[:, None, None] * freq
    c, s = angle.cos().float(), angle.sin().float()
    q, k = (torch.cat([t[..., :D // 2] * c - t[..., D // 2:] * s, t[..., D // 2:] * c + t[..., :D // 2] * s], -1) for t in (q, k))
    k, v = (t.repeat_interleave(heads // kv_heads, 1) for t in (k, v))
    p = torch.softmax((q[-1][None] * k).sum(-1) * D ** -0.5, 0)
    return (p[..., None] * v).sum(0).reshape(1, -1) @ wo.T


def run(kind="i8", hidden=1024, heads=8, kv_heads=2, counts=(130, 1, 57), steps=5, report=print):
    kv = kv_heads * hidden // heads
    made = [random_weights(n, hidden, seed) for seed, n in enumerate((hidden, kv, kv, hidden))]
    block = AttentionBlock(hidden, heads, kv_heads, [m[0] for m in made], kind, len(counts), max(counts) + steps)
    torch.manual_seed(1)
    prompts = [torch.randn((n, hidden), device="cuda").half() for n in counts]
    ticks = [torch.cuda.Event(enable_timing=True) for _ in range(3)]
    ticks[0].record()
    block.prefill(torch.cat(prompts), counts)
    ticks[1].record()
    for _ in range(steps):
        x = torch.randn((len(counts), hidden), device="cuda").half()
        y = block.step(x)
        prompts = [torch.cat([p, x[b:b + 1]]) for b, p in enumerate(prompts)]
    ticks[2].record()
    torch.cuda.synchronize()
    want = torch.cat([dense_last(p.float(), [m[1] for m in made], heads, kv_heads) for p in prompts])
    error = ((y.float() - want).norm() / want.norm()).item()
    report(f"prefill of {sum(counts)} tokens {ticks[0].elapsed_time(ticks[1]):.3f} ms, {steps} steps "
           f"{ticks[1].elapsed_time(ticks[2]):.3f} ms, cache {kind}: last step {error:.2e} off the dense block")
    return error


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--kind", default="i8", choices=("f16", "i8", "i4"))
    ap.add_argument("--hidden", type=int, default=1024)
    ap.add_argument("--heads", type=int, default=8)
    ap.add_argument("--kv-heads", type=int, default=2)
    a = ap.parse_args()
    run(a.kind, a.hidden, a.heads, a.kv_heads)
