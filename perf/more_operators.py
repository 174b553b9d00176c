"""A decoder layer on 4-bit weights, operator by operator, as cases to be timed and compared.

Around the attention block a layer normalises its hidden state, multiplies it by packed weights, and gates the products
of its feed-forward half.  The sizes are those of the 7B (hidden 4096, 11008 wide) and 70B (8192, 28672) decoders, and in
draw() generic ones around them.

op norm     h = x + r (the residual stream), y = h / sqrt(mean(h^2) + eps) * w, for M tokens; h comes back too
op gate     act(gate) * up for M tokens: silu, or gelu by its tanh form
op product  y = x W^T for one to three weights W that read the same x: 16-bit x, or signed bytes and a scale a token
op block    norm and the products after it, as at the head of an attention block; i8: the norm's output in 8 bits
op mlp      norm, gate and up products, their gating, the down product; i8: norm and gating give 8 bits

4-bit weights.  W[n][k] = scale[n][k / 128] * (code[n][k] - 8), codes 0 to 15, scales f16.  Packed: for every 16 rows and
128 columns 64 slots of 16 bytes, slot s = row s % 16 and columns 64 (j / 2) + 16 (s / 16) + 8 (j % 2) .. + 7 for the words
j = 0 .. 3, byte b of a word holding column b in its low half and column 4 + b in its high half; after all codes, for every
16 rows and 4 groups, 8 bytes a row with the groups' scales (zeros behind the last group).
8 bits.  A token's values are code * scale, scale = a / 127 with a the token's largest magnitude, code = round(v / scale).
"""
import math
import random

import torch

own = False

DTYPE = {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}
GROUP = 128
EPS = 1e-5


# ---------------------------------------------------------------- cases

def _norm(M, n, dtype="f16", stream="", weight=""):
    """stream, weight: the types of the residual stream and of the weights (x's where not said)."""
    return {"op": "norm", "M": M, "n": n, "dtype": dtype, "stream": stream or dtype, "weight": weight or dtype}


def _gate(M, n, dtype="f16", act="silu"):
    return {"op": "gate", "M": M, "n": n, "dtype": dtype, "act": act}


def _product(M, K, N0, N1=0, N2=0, dtype="f16", i8=False, out=""):
    return {"op": "product", "M": M, "K": K, "N0": N0, "N1": N1, "N2": N2, "dtype": dtype, "i8": i8, "out": out or dtype}


def _block(M, K, N0, N1, N2, dtype="f16", i8=True):
    return {"op": "block", "M": M, "K": K, "N0": N0, "N1": N1, "N2": N2, "dtype": dtype, "i8": i8}


def _mlp(M, K, F, dtype="f16", i8=True, act="silu"):
    return {"op": "mlp", "M": M, "K": K, "F": F, "dtype": dtype, "i8": i8, "act": act}


def listed():
    return [
        # a decoding step of one sequence: latency only
        dict(_norm(1, 4096), name="norm_7b_m1"),
        # a packed batch of prompts on a residual stream of 32 bits
        dict(_norm(4096, 8192, "bf16", "f32"), name="norm_70b_m4096"),
        # a decoding step of 16 sequences
        dict(_gate(16, 11008), name="gate_7b_m16"),
        # a prompt's feed-forward half
        dict(_gate(2048, 28672, "bf16"), name="gate_70b_m2048"),
        # one token through one layer's output product
        dict(_product(1, 4096, 4096), name="product_7b_m1"),
        # four drafted tokens through gate and up
        dict(_product(4, 4096, 11008, 11008, dtype="bf16"), name="product_7b_m4"),
        # 16 sequences in 8 bits through the down product, the longest rows
        dict(_product(16, 28672, 8192, dtype="bf16", i8=True), name="product_70b_m16_i8"),
        # 61 sequences through q, k and v with grouped heads
        dict(_product(61, 8192, 8192, 1024, 1024), name="product_70b_m61"),
        # a prompt through gate and up
        dict(_product(2048, 4096, 11008, 11008, dtype="bf16"), name="product_7b_m2048"),
        # the same in 8 bits
        dict(_product(2048, 4096, 11008, 11008, dtype="bf16", i8=True), name="product_7b_m2048_i8"),
        # a short prompt of odd length into an attention block, in 8 bits
        dict(_block(333, 4096, 4096, 4096, 4096, "bf16"), name="block_7b_m333_i8"),
        # one token through the whole feed-forward half: five launches' latency and the weights' read
        dict(_mlp(1, 8192, 28672, i8=False), name="mlp_70b_m1"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["norm", "gate", "product", "product", "product", "product", "block", "mlp"])
    dtype = rng.choice(["f16", "bf16"])
    if op in ("norm", "gate"):
        n = 8 * _log(rng, 8, 3584)
        M = _log(rng, 1, max(2, 4096 * 8192 // n))
        if op == "norm":
            return _norm(M, n, dtype, rng.choice([dtype, "f32"]), rng.choice([dtype, "f32"]))
        return _gate(M, n, dtype, rng.choice(["silu", "silu", "gelu"]))
    K = GROUP * _log(rng, 1, 86)
    N = 16 * _log(rng, 1, 688)
    M = min(_log(rng, 1, 3000), int(1.8e11 / (K * N * 2)) + 1)
    i8 = rng.random() < 0.4
    if op == "mlp":
        F = GROUP * _log(rng, 2, 172)
        while M * K * F > 3e10:
            M = max(1, M * 2 // 3)
        return _mlp(M, K, F, dtype, i8, rng.choice(["silu", "silu", "gelu"]))
    N1, N2 = rng.choice([(0, 0), (0, 0), (N, 0), (16 * _log(rng, 1, 64), 16 * _log(rng, 1, 64))])
    while M * K * (N + N1 + N2) > 9e10:
        M = max(1, M * 2 // 3)
    if op == "block":
        return _block(M, K, N, N1, N2, dtype, i8)
    return _product(M, K, N, N1, N2, dtype, i8, rng.choice([dtype, dtype, "f32"]))


# ---------------------------------------------------------------- inputs

def _weights(N, K, gen):
    """Codes uint8 [N][K], scales f16 [N][K / 128] and both packed."""
    groups, dev = K // GROUP, gen.device
    codes = torch.randn((N, K), generator=gen, device=dev).mul_(2.4).add_(8.0).round_().clamp_(0, 15).to(torch.uint8)
    scales = ((torch.rand((N, groups), generator=gen, device=dev) + 0.5) * (0.4 / math.sqrt(K))).to(torch.float16)
    # [rows of 16][row][group][word j / 2][chunk][j % 2][half][byte] -> [rows of 16][group][chunk][row][j / 2][j % 2][byte][half]
    c = codes.view(N // 16, 16, groups, 2, 4, 2, 2, 4).permute(0, 2, 4, 1, 3, 5, 7, 6)
    body = (c[..., 0] | c[..., 1] << 4).reshape(-1)
    quads = -(-groups // 4)
    tail = torch.zeros((N, 4 * quads), dtype=torch.float16, device=dev)
    tail[:, :groups] = scales
    tail = tail.view(N // 16, 16, quads, 4).transpose(1, 2).contiguous().view(torch.uint8).reshape(-1)
    return {"N": N, "K": K, "codes": codes, "scales": scales, "packed": torch.cat([body, tail])}


def _hidden(M, n, dtype, gen):
    """Activations with a few channels that are much larger than the others, as hidden states have them."""
    x = torch.randn((M, n), generator=gen, device=gen.device)
    x *= torch.where(torch.rand(n, generator=gen, device=gen.device) < 0.01, 20.0, 1.0)
    return x.to(dtype)


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    op, M, dtype = case["op"], case["M"], DTYPE[case["dtype"]]
    s = {"case": case}
    if op == "gate":
        s["gate"], s["up"] = (_hidden(M, case["n"], dtype, gen) for _ in range(2))
        return s
    n = case["n"] if op == "norm" else case["K"]
    if op == "product" and case["i8"]:
        v = _hidden(M, n, torch.float32, gen)
        scale = v.abs().amax(1) / 127.0
        s["x"] = (v / scale[:, None]).round().clamp(-127, 127).to(torch.int8), scale
    else:
        s["x"] = _hidden(M, n, dtype, gen)
    if op != "product":
        s["residual"] = _hidden(M, n, DTYPE[case["stream"]] if op == "norm" else dtype, gen)
        w = 1.0 + 0.1 * torch.randn(n, generator=gen, device=gen.device)
        s["norm"] = w.to(DTYPE[case["weight"]] if op == "norm" else dtype)
    if op == "mlp":
        s["weights"] = [_weights(case["F"], n, gen) for _ in range(2)]
        s["down"] = _weights(n, case["F"], gen)
    elif op != "norm":
        s["weights"] = [_weights(N, n, gen) for N in (case["N0"], case["N1"], case["N2"]) if N]
    return s


# ---------------------------------------------------------------- plain form

def _plain_norm(s):
    """The residual stream after the addition, and the normalised rows in 32 bits."""
    h = (s["x"].float() + s["residual"].float()).to(s["residual"].dtype)
    f = h.float()
    return h, f * torch.rsqrt((f * f).mean(1, keepdim=True) + EPS) * s["norm"].float()


def _plain_gate(gate, up, act):
    g = gate.float()
    if act == "gelu":
        return 0.5 * g * (1.0 + torch.tanh(math.sqrt(2.0 / math.pi) * (g + 0.044715 * g * g * g))) * up.float()
    return g / (1.0 + torch.exp(-g)) * up.float()


def _plain_bytes(v):
    """What 32-bit rows are once they are held in 8 bits."""
    scale = v.abs().amax(1, keepdim=True) / 127.0
    return torch.round(v * (1.0 / scale)).clamp(-127, 127) * scale


def _plain_product(x, w, dtype):
    dense = (w["codes"].float() - 8.0).view(w["N"], -1, GROUP) * w["scales"].float()[:, :, None]
    return (x.float() @ dense.view(w["N"], w["K"]).T).to(dtype)


def _plain(s):
    case = s["case"]
    op, dtype = case["op"], DTYPE[case["dtype"]]
    if op == "gate":
        return _plain_gate(s["gate"], s["up"], case["act"]).to(dtype)
    if op == "product":
        x = s["x"][0].float() * s["x"][1][:, None] if case["i8"] else s["x"]
        return [_plain_product(x, w, DTYPE[case["out"]]) for w in s["weights"]]
    h, y = _plain_norm(s)
    if op == "norm":
        return {"h": h, "y": y.to(dtype)}
    y = _plain_bytes(y) if case["i8"] else y.to(dtype)
    outs = [_plain_product(y, w, dtype) for w in s["weights"]]
    if op == "block":
        return {"h": h, "outs": outs}
    a = _plain_gate(*outs, case["act"])
    return {"h": h, "y": _plain_product(_plain_bytes(a) if case["i8"] else a.to(dtype), s["down"], dtype)}


# ---------------------------------------------------------------- the framework's kernels

def _own(s):
    import paper_2606_10520_amd.unisvq as u
    case = s["case"]
    op, dtype = case["op"], DTYPE[case["dtype"]]
    if op == "gate":
        return u.gated(s["gate"], s["up"], case["act"])
    if op == "norm":
        y, h = u.rmsnorm(s["x"], s["norm"], EPS, residual=s["residual"])
        return {"h": h, "y": y}
    if op == "product":
        if len(s["weights"]) == 1:
            w = s["weights"][0]
            return [u.fourbit_gemm(w["packed"], w["N"], w["K"], s["x"], out_dtype=DTYPE[case["out"]])]
        return u.fourbit_gemm_batched([(w["packed"], w["N"], w["K"], s["x"], None) for w in s["weights"]],
                                 out_dtype=DTYPE[case["out"]])
    kept = torch.int8 if case["i8"] else dtype
    y, h = u.rmsnorm(s["x"], s["norm"], EPS, residual=s["residual"], out_dtype=kept)
    outs = u.fourbit_gemm_batched([(w["packed"], w["N"], w["K"], y, None) for w in s["weights"]], out_dtype=dtype)
    if op == "block":
        return {"h": h, "outs": outs}
    a = u.gated(*outs, case["act"], out_dtype=kept)
    w = s["down"]
    return {"h": h, "y": u.fourbit_gemm(w["packed"], w["N"], w["K"], a, out_dtype=dtype)}


def run(state):
    return _own(state) if own else _plain(state)


# ---------------------------------------------------------------- what a pass cannot do without

def _weight_bytes(N, K):
    return N * K // 2 + N * (K // GROUP) * 2


def work(case):
    op, M = case["op"], case["M"]
    size = 4 if case["dtype"] == "f32" else 2
    if op == "gate":
        return {"bytes": 3 * M * case["n"] * size, "flops": 8 * M * case["n"]}
    if op == "norm":
        n, stream = case["n"], 4 if case["stream"] == "f32" else 2
        return {"bytes": M * n * (2 * size + 2 * stream) + n * (4 if case["weight"] == "f32" else 2), "flops": 6 * M * n}
    K = case["K"]
    if op == "mlp":
        F = case["F"]
        return {"bytes": 4 * M * K * size + 2 * K + 2 * _weight_bytes(F, K) + _weight_bytes(K, F),
                "flops": 6 * M * K * F}
    rows = [N for N in (case["N0"], case["N1"], case["N2"]) if N]
    flops, read = 2 * M * K * sum(rows), sum(_weight_bytes(N, K) for N in rows)
    if op == "block":
        return {"bytes": 3 * M * K * size + 2 * K + read + M * sum(rows) * size, "flops": flops}
    return {"bytes": (M * K + 4 * M if case["i8"] else M * K * size) + read + M * sum(rows) * (4 if case["out"] == "f32" else 2),
            "flops": flops}


# ---------------------------------------------------------------- 64 bits

def _exact_rows(x, w):
    """x W^T of 64-bit rows x, group by group of columns."""
    y = torch.zeros((x.shape[0], w["N"]), dtype=torch.float64, device=x.device)
    for g in range(w["K"] // GROUP):
        cols = slice(g * GROUP, (g + 1) * GROUP)
        y += (x[:, cols] @ (w["codes"][:, cols].double() - 8.0).T) * w["scales"][:, g].double()
    return y


def _exact_bytes(v):
    top = v.abs().max(dim=1, keepdim=True).values
    return torch.round(v * 127.0 / top) * top / 127.0


def _exact_gate(g, u, act):
    if act == "gelu":
        t = math.sqrt(8.0 / math.pi) * (g + 0.044715 * g ** 3)
        return g * u / (1.0 + torch.exp(-t))  # (1 + tanh(t / 2)) / 2 = 1 / (1 + exp(-t))
    return g * u * torch.sigmoid(g)


def exact(case, seed):
    s = prepare(case, seed)
    op, dtype = case["op"], DTYPE[case["dtype"]]
    if op == "gate":
        return _exact_gate(s["gate"].double(), s["up"].double(), case["act"])
    if op == "product":
        x = s["x"][0].double() * s["x"][1].double()[:, None] if case["i8"] else s["x"].double()
        return [_exact_rows(x, w) for w in s["weights"]]
    wide = s["x"].double() + s["residual"].double()
    h = wide.to(s["residual"].dtype).double()  # the stream as it is kept is what is normalised
    y = h / torch.sqrt(h.square().sum(1, keepdim=True) / h.shape[1] + EPS) * s["norm"].double()
    if op == "norm":
        return {"h": wide, "y": y}
    y = _exact_bytes(y) if case["i8"] else y.to(dtype).double()
    outs = [_exact_rows(y, w) for w in s["weights"]]
    if op == "block":
        return {"h": wide, "outs": outs}
    a = _exact_gate(*(o.to(dtype).double() for o in outs), case["act"])
    return {"h": wide, "y": _exact_rows(_exact_bytes(a) if case["i8"] else a.to(dtype).double(), s["down"])}
