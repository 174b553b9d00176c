"""A whole decoder layer, served on 4-bit weights: norm, q/k/v products, rotary positions, cache and attention, o product, norm,
gate and up products, gated activation, down product, with the residual stream added on the way.  A batch of prompts of
different lengths goes through in one pass, then tokens are generated one at a time.

    python examples/decoder_layer.py [--kind i8] [--eight] [--hidden 1024] [--heads 8] [--kv-heads 2] [--width 2816]

--eight: activations of the q/k/v, gate/up and down products in 8 bits.  Prints the time of both and how far the last step is
from the same step computed densely in fp32 with the same (rounded) weights.
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2606_10520_amd.unisvq as u  # noqa: E402

EPS = 1e-5


class DecoderLayer:
    """(x, stream) -> (y, stream): x is what the layer before gave, to be added to the residual stream; y is this layer's."""

    def __init__(self, weights, heads, kv_heads, kind, sequences, max_len, eight=False, page_tokens=64):
        self.w, self.shape = {}, {}
        for name in ("q", "k", "v", "o", "gate", "up", "down"):
            self.shape[name] = weights[name].shape
            self.w[name] = u.fourbit_quantize(weights[name])
        self.norm1, self.norm2 = weights["norm1"], weights["norm2"]
        self.hidden = weights["q"].shape[1]
        self.heads, self.kv_heads, self.D = heads, kv_heads, weights["q"].shape[0] // heads
        self.kept = torch.int8 if eight else None
        width = -(-max_len // page_tokens)
        self.cache = u.new_cache(sequences * width, kv_heads, page_tokens, self.D, kind)
        self.pages = torch.randperm(sequences * width, device="cuda").to(torch.int32).view(sequences, width)
        self.lens = torch.zeros(sequences, dtype=torch.int32, device="cuda")
        self.rope = u.rope_table(max_len, self.D)

    def _products(self, x, *names):
        return u.fourbit_gemm_batched([(self.w[n], *self.shape[n], x, None) for n in names], out_dtype=torch.float16)

    def _qkv(self, x, stream):
        y, _ = u.rmsnorm(x, self.norm1, EPS, residual=stream, residual_out=stream, out_dtype=self.kept)
        return (t.view(x.shape[0], -1, self.D) for t in self._products(y, "q", "k", "v"))

    def _rest(self, o, stream):
        x = self._products(o.view(o.shape[0], -1), "o")[0]
        y, _ = u.rmsnorm(x, self.norm2, EPS, residual=stream, residual_out=stream, out_dtype=self.kept)
        return self._products(u.gated(*self._products(y, "gate", "up"), out_dtype=self.kept), "down")[0]

    def prefill(self, x, stream, counts):
        """x, stream [tokens][hidden]: counts[b] new tokens of every sequence b, after what its cache holds."""
        n = torch.tensor(counts, dtype=torch.int32, device=x.device)
        zero = torch.zeros(1, dtype=torch.int32, device=x.device)
        seqs = torch.repeat_interleave(torch.arange(len(counts), device=x.device), n.long()).to(torch.int32)
        cu_q = torch.cat([zero, n.cumsum(0).to(torch.int32)])
        positions = (torch.arange(x.shape[0], device=x.device) - cu_q[seqs.long()] + self.lens[seqs.long()]).to(torch.int32)
        q, k, v = self._qkv(x, stream)
        q = u.cache_append(self.cache, self.pages, seqs, positions, k, v, q=q, rope_table=self.rope, q_out=q)
        self.lens += n
        cu_k = torch.cat([zero, self.lens.cumsum(0).to(torch.int32)])
        k, v = u.cache_read(self.cache, self.pages, None, cu_k, int(cu_k[-1]), out_dtype=x.dtype)
        return self._rest(u.attn_prompt(q, k, v, cu_q, cu_k), stream)

    def step(self, x, stream):
        """x, stream [sequences][hidden]: the next token of every sequence."""
        q, k, v = self._qkv(x, stream)
        q = u.cache_append(self.cache, self.pages, None, self.lens, k, v, q=q, rope_table=self.rope, q_out=q)
        self.lens += 1
        return self._rest(u.attn_decode(q, self.cache, self.pages, self.lens), stream)


def random_weights(hidden, heads, kv_heads, width, seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    D = hidden // heads
    rows = {"q": (hidden, hidden), "k": (kv_heads * D, hidden), "v": (kv_heads * D, hidden), "o": (hidden, hidden),
            "gate": (width, hidden), "up": (width, hidden), "down": (hidden, width)}
    w = {n: (torch.randn(s, generator=g, device="cuda") * s[1] ** -0.5).half() for n, s in rows.items()}
    for n in ("norm1", "norm2"):
        w[n] = (1 + 0.1 * torch.randn(hidden, generator=g, device="cuda")).half()
    return w


def dense(layer, name):
    """The layer's weights as they were rounded, in fp32."""
    codes, scales = u.fourbit_unpack(layer.w[name], *layer.shape[name])
    return ((codes.float() - 8).view(*scales.shape, 128) * scales.float()[..., None]).view(codes.shape)


def dense_last(layer, x, stream):
    """The layer's output for the last token of one sequence x, stream [tokens][hidden], in fp32."""
    w = {n: dense(layer, n) for n in layer.w}
    n, D = x.shape[0], layer.D

    def norm(h, weight):
        return h * torch.rsqrt(h.square().mean(1, keepdim=True) + EPS) * weight.float()

    h = x + stream
    y = norm(h, layer.norm1)
    q, k, v = ((y @ w[t].T).view(n, -1, D) for t in "qkv")
    freq = 10000.0 ** (-torch.arange(0, D, 2, dtype=torch.float64, device=x.device) / D)
    angle = torch.arange(n, dtype=torch.float64, device=x.device)[:, None, None] * freq
    c, s = angle.cos().float(), angle.sin().float()
    q, k = (torch.cat([t[..., :D // 2] * c - t[..., D // 2:] * s, t[..., D // 2:] * c + t[..., :D // 2] * s], -1) for t in (q, k))
    k, v = (t.repeat_interleave(layer.heads // layer.kv_heads, 1) for t in (k, v))
    p = torch.softmax((q[-1][None] * k).sum(-1) * D ** -0.5, 0)
    h = h[-1:] + (p[..., None] * v).sum(0).reshape(1, -1) @ w["o"].T
    y = norm(h, layer.norm2)
    return (torch.nn.functional.silu(y @ w["gate"].T) * (y @ w["up"].T)) @ w["down"].T


def run(kind="i8", eight=False, hidden=1024, heads=8, kv_heads=2, width=2816, counts=(130, 1, 57), steps=5, report=print):
    layer = DecoderLayer(random_weights(hidden, heads, kv_heads, width), heads, kv_heads, kind, len(counts), max(counts) + steps, eight)
    torch.manual_seed(1)
    xs = [torch.randn((n, hidden), device="cuda").half() for n in counts]
    streams = [torch.randn((n, hidden), device="cuda").half() for n in counts]
    ticks = [torch.cuda.Event(enable_timing=True) for _ in range(3)]
    ticks[0].record()
    layer.prefill(torch.cat(xs), torch.cat(streams), counts)
    ticks[1].record()
    for _ in range(steps):
        x, stream = (torch.randn((len(counts), hidden), device="cuda").half() for _ in range(2))
        xs = [torch.cat([p, x[b:b + 1]]) for b, p in enumerate(xs)]
        streams = [torch.cat([p, stream[b:b + 1]]) for b, p in enumerate(streams)]
        y = layer.step(x, stream)
    ticks[2].record()
    torch.cuda.synchronize()
    want = torch.cat([dense_last(layer, p.float(), s.float()) for p, s in zip(xs, streams)])
    error = ((y.float() - want).norm() / want.norm()).item()
    report(f"prefill of {sum(counts)} tokens {ticks[0].elapsed_time(ticks[1]):.3f} ms, {steps} steps "
           f"{ticks[1].elapsed_time(ticks[2]):.3f} ms, cache {kind}, activations of {8 if eight else 16} bits: "
           f"last step {error:.2e} off the dense layer")
    return error


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--kind", default="i8", choices=("f16", "i8", "i4"))
    ap.add_argument("--eight", action="store_true")
    ap.add_argument("--hidden", type=int, default=1024)
    ap.add_argument("--heads", type=int, default=8)
    ap.add_argument("--kv-heads", type=int, default=2)
    ap.add_argument("--width", type=int, default=2816)
    a = ap.parse_args()
    run(a.kind, a.eight, a.hidden, a.heads, a.kv_heads, a.width)
