"""The attention block of a served decoder, operator by operator, as cases to be timed and compared.

Between the q/k/v product of a decoder layer and its o product a serving program rotates q and k to their positions,
writes k and v to a paged cache (as they are, or quantised to 8 or 4 bits), and attends: to the prompt's own tokens, or,
for the tokens being generated, to the cache.  The sizes are those of the 7B (32 heads) and 70B (64 query heads on 8
key/value heads) decoders, and in draw() generic ones around them.

op rope    q or k of T tokens rotated by a table of cosines and sines at each token's position; inverse: the gradient
op cache   q, k, v of `new` tokens a sequence: q rotated, k rotated and stored, v stored; then tokens read back
           (read_all: the whole sequence, as a chunk of a prompt needs it; else the tokens just written)
op decode  q_len new tokens of each of B sequences against the cache
op prompt  packed sequences of `len` tokens, each after `ctx` tokens that are there already

What the cache holds.  Pools [pages][kv_heads][page][D] (page: tokens of a page), 4-bit codes two to a byte (the even
dim in the low half), and a table [B][pages of a sequence].  kind f16 / bf16: the values; i8: signed codes and one f32
scale a token and head, a / 127 with a the largest magnitude; i4: codes + 8 and two bf16 scales a token and head, a / 7
for each half of the head.  code = round(x * (1 / scale)), clamped; the scale is 0 where a < 1e-30, NaN where x is not finite.
"""
import math
import random

import torch

own = False

DTYPE = {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}


# ---------------------------------------------------------------- cases

def _rope(T, heads, D=128, rot=None, layout="half", inverse=False, dtype="f16", max_pos=4096, factor=1.0):
    return {"op": "rope", "T": T, "heads": heads, "D": D, "rot": rot or D, "layout": layout, "inverse": inverse,
            "dtype": dtype, "max_pos": max_pos, "factor": factor}


def _cache(B, new, ctx, q_heads, kv_heads, D=128, page=64, kind="i8", dtype="f16", rot=None, layout="half",
           ragged=False, read_all=False):
    return {"op": "cache", "B": B, "new": new, "ctx": ctx, "q_heads": q_heads, "kv_heads": kv_heads, "D": D,
            "page": page, "kind": kind, "dtype": dtype, "rot": rot or D, "layout": layout, "ragged": ragged,
            "read_all": read_all}


def _decode(B, length, q_heads, kv_heads, q_len=1, D=128, page=64, kind="i8", dtype="f16", ragged=False):
    return {"op": "decode", "B": B, "len": length, "q_len": q_len, "q_heads": q_heads, "kv_heads": kv_heads, "D": D,
            "page": page, "kind": kind, "dtype": dtype, "ragged": ragged}


def _prompt(B, length, ctx, q_heads, kv_heads, D=128, dtype="bf16", ragged=False, causal=True):
    return {"op": "prompt", "B": B, "len": length, "ctx": ctx, "q_heads": q_heads, "kv_heads": kv_heads, "D": D,
            "dtype": dtype, "ragged": ragged, "causal": causal}


def listed():
    return [
        # the smallest call: q of four sequences' next tokens, latency only
        dict(_rope(4, 32), name="rope_7b_m4"),
        # the gradient of a long packed batch's q: interleaved pairs in half of the head, positions stretched 8 times
        dict(_rope(8192, 64, rot=64, layout="interleaved", inverse=True, dtype="bf16", max_pos=65536, factor=8.0),
             name="rope_70b_grad_m8192"),
        # a decoding step of 16 sequences: rotate q and k, write one token each
        dict(_cache(16, 1, 1000, 32, 32), name="cache_7b_step_b16"),
        # a prompt written to the 8-bit cache and handed back for its attention
        dict(_cache(1, 2048, 0, 64, 8, dtype="bf16", read_all=True), name="cache_70b_m2048"),
        # a chunk of each of four prompts of different lengths into a 4-bit cache of small pages, all of it read back
        dict(_cache(4, 500, 1000, 32, 32, page=16, kind="i4", layout="interleaved", ragged=True, read_all=True),
             name="cache_7b_chunk_i4"),
        # one sequence, a cache of plain f16 values, an odd length: latency and a long axis to split
        dict(_decode(1, 1001, 32, 32, kind="f16"), name="decode_7b_b1"),
        # a ragged batch with grouped heads on the 8-bit cache, one slot of the batch empty
        dict(_decode(16, 8192, 64, 8, dtype="bf16", ragged=True), name="decode_70b_b16"),
        # long sequences in the 4-bit cache: the largest read
        dict(_decode(4, 32768, 32, 32, page=32, kind="i4"), name="decode_7b_b4_i4"),
        # the prompt of the 7B decoder
        dict(_prompt(1, 2048, 0, 32, 32), name="prompt_7b_m2048"),
        # prompts of different lengths in one call, from one token on, grouped heads
        dict(_prompt(8, 1500, 0, 64, 8, dtype="f16", ragged=True), name="prompt_70b_packed"),
        # chunks of four prompts after what was cached of them: few rows, many keys
        dict(_prompt(4, 256, 3000, 64, 8, ragged=True), name="prompt_70b_chunk"),
        # a long prompt: the largest product
        dict(_prompt(1, 16384, 0, 32, 32), name="prompt_7b_m16384"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["rope", "cache", "decode", "decode", "decode", "prompt", "prompt", "prompt"])
    D = rng.choice([128, 128, 128, 64])
    kv = rng.choice([2, 4, 8, 8, 16, 32])
    q = kv * rng.choice([1, 1, 2, 4, 5, 8]) if kv <= 8 else kv * rng.choice([1, 2])
    dtype = rng.choice(["f16", "bf16"])
    layout = rng.choice(["half", "half", "interleaved"])
    rot = rng.choice([D, D, D // 2, D // 2 + 16])
    page = rng.choice([16, 32, 64, 128, 256])
    kind = rng.choice([dtype, "i8", "i8", "i4"])
    if op == "rope":
        return _rope(_log(rng, 1, 8192 * 64 // max(q, 64)), q, D, rot, layout, rng.random() < 0.3, dtype,
                     _log(rng, 2048, 131072), rng.choice([1.0, 1.0, 4.0, 16.0]))
    if op == "cache":
        if rng.random() < 0.5:
            return _cache(rng.randint(1, 64), rng.randint(1, 4), _log(rng, 1, 4000), q, kv, D, page, kind, dtype, rot,
                          layout, rng.random() < 0.5, False)
        B = rng.randint(1, 5)
        new = _log(rng, 17, 2048 // B)
        return _cache(B, new, rng.choice([0, _log(rng, 1, 2000)]), q, kv, D, page, kind, dtype, rot, layout,
                      B > 1 and rng.random() < 0.7, True)
    if op == "decode":
        B = _log(rng, 1, 64)
        most = int(500e6 / (B * kv * D * {"i8": 2.1, "i4": 1.1}.get(kind, 4.0)))
        return _decode(B, _log(rng, 1, max(2, min(32768, most))), q, kv, rng.choice([1, 1, 1, 2, 4]), D, page, kind,
                       dtype, B > 1 and rng.random() < 0.7)
    B = rng.choice([1, 1, 2, 3, 5, 9])
    if rng.random() < 0.3:
        length, ctx = _log(rng, 1, 600 // B + 1), _log(rng, 1, 4000)
    else:
        length, ctx = _log(rng, 16, min(8192, 12000 // B)), 0
    # the plain form holds all scores of the packed batch
    most = 24e9 / 4 / q
    while B * length * B * (length + ctx) > most:
        length, ctx = max(1, length * 4 // 5), ctx * 4 // 5
    return _prompt(B, length, ctx, q, kv, D, dtype, B > 1 and rng.random() < 0.7, rng.random() < 0.85)


def _lens(B, most, ragged, least=0):
    """The lengths of a batch's sequences, up to `most`, which one of them has; where ragged and the batch is large, one is the least."""
    if not ragged:
        return [most] * B
    r = random.Random(B * 1000003 + most)
    lens = [max(least, min(most, int(math.exp(r.uniform(math.log(max(most, 64) / 64), math.log(most + 1)))))) for _ in range(B)]
    lens[r.randrange(B)] = most
    if B >= 8:
        lens[(lens.index(most) + 1) % B] = least
    return lens


# ---------------------------------------------------------------- inputs

def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _randn(g, *shape, dtype=torch.float32, std=1.0):
    return (torch.randn(shape, generator=g, device="cuda") * std).to(dtype)


def _ints(v, dtype=torch.int32):
    return torch.tensor(v, dtype=dtype, device="cuda")


def _cum(lens):
    out = [0]
    for n in lens:
        out.append(out[-1] + n)
    return out


def _table(positions, rot, factor=1.0, theta=10000.0):
    """Cosines and sines [positions][2][rot / 2]; positions stretched by `factor` (linear scaling for long contexts)."""
    freq = theta ** (-torch.arange(0, rot, 2, dtype=torch.float64, device="cuda") / rot) / factor
    angle = torch.arange(positions, dtype=torch.float64, device="cuda")[:, None] * freq
    return torch.stack([angle.cos(), angle.sin()], 1).float().contiguous()


def _pools(g, case, lens):
    """Pools that hold `lens` tokens of each sequence, their pages in no order; what no token has written is garbage."""
    B, page, H, D, kind = case["B"], case["page"], case["kv_heads"], case["D"], case["kind"]
    need = [-(-n // page) for n in lens]
    width = max(1, max(need))
    pages = max(1, sum(need))
    order = torch.randperm(pages, generator=g, device="cuda", dtype=torch.int64).to(torch.int32)
    table = torch.full((B, width), -1, dtype=torch.int32, device="cuda")
    at = _cum(need)
    for b in range(B):
        table[b, : need[b]] = order[at[b]: at[b + 1]]
    shape = (pages, H, page)
    scales = [None, None]
    if kind in ("f16", "bf16"):
        kv = [_randn(g, *shape, D, dtype=DTYPE[kind]) for _ in range(2)]
    elif kind == "i8":
        kv = [_randn(g, *shape, D, std=42.0).round_().clamp_(-127, 127).to(torch.int8) for _ in range(2)]
        scales = [torch.rand(shape, generator=g, device="cuda") * 0.012 + 0.018 for _ in range(2)]
    else:
        half = [torch.randint(1, 16, (*shape, D // 2), generator=g, device="cuda", dtype=torch.uint8) for _ in range(4)]
        kv = [half[0] | half[1] << 4, half[2] | half[3] << 4]
        scales = [(torch.rand((*shape, 2), generator=g, device="cuda") * 0.1 + 0.2).to(torch.bfloat16) for _ in range(2)]
    # the places past a sequence's end
    pos = torch.arange(width * page, device="cuda").reshape(width, page)
    for b in range(B):
        if need[b] and lens[b] % page:
            free = (pos[need[b] - 1] >= lens[b])[None, :].expand(H, page)
            p = int(at[b + 1] - 1)
            for x in (kv if kind in ("f16", "bf16") else scales):
                x[int(order[p])][free] = float("nan")
    return {"k": kv[0], "v": kv[1], "ks": scales[0], "vs": scales[1], "table": table}


def prepare(case, seed):
    g = _gen(seed)
    s = {"case": case}
    D = case["D"]
    dtype = DTYPE[case["dtype"]]
    if case["op"] == "rope":
        T = case["T"]
        s["table"] = _table(case["max_pos"], case["rot"], case["factor"])
        s["x"] = _randn(g, T, case["heads"], D, dtype=dtype)
        # next tokens are anywhere; the tokens of prompts follow each other, from any position on
        r = random.Random(seed)
        start = r.randrange(max(1, case["max_pos"] - T))
        s["pos"] = (_ints([r.randrange(case["max_pos"]) for _ in range(T)]) if T <= 64
                    else (torch.arange(T, device="cuda") + start).remainder(case["max_pos"]).to(torch.int32))
        s["out"] = torch.empty_like(s["x"])
    elif case["op"] == "cache":
        B, new, Hq, H = case["B"], case["new"], case["q_heads"], case["kv_heads"]
        before = _lens(B, case["ctx"], case["ragged"])
        lens = [n + new for n in before]
        T = B * new
        s.update(_pools(g, case, lens))
        s["rope"] = _table(max(lens), case["rot"])
        s["qkv"] = _randn(g, T, Hq + 2 * H, D, dtype=dtype)
        s["qkv"][:, :, torch.randperm(D, generator=g, device="cuda")[: D // 64]] *= 5  # channels that stand out
        s["q"], s["knew"], s["vnew"] = s["qkv"].split([Hq, H, H], dim=1)
        s["seq"] = torch.arange(B, device="cuda").repeat_interleave(new).to(torch.int32)
        s["pos"] = (_ints(before)[:, None] + torch.arange(new, device="cuda")).reshape(-1).to(torch.int32)
        s["start"] = _ints([0] * B if case["read_all"] else before)
        s["total"] = sum(lens) if case["read_all"] else T
        s["cu"] = _ints(_cum(lens if case["read_all"] else [new] * B))
        s["q_out"] = torch.empty((T, Hq, D), dtype=dtype, device="cuda")
        s["k_out"] = torch.empty((s["total"], H, D), dtype=dtype, device="cuda")
        s["v_out"] = torch.empty_like(s["k_out"])
    elif case["op"] == "decode":
        lens = _lens(case["B"], case["len"], case["ragged"])
        s.update(_pools(g, case, lens))
        s["lens"] = _ints(lens)
        s["q"] = _randn(g, case["B"], case["q_len"], case["q_heads"], D, dtype=dtype, std=2.0)
        s["out"] = torch.empty_like(s["q"])
        s["lse"] = torch.empty(s["q"].shape[:3], device="cuda")
    else:
        B, Hq, H = case["B"], case["q_heads"], case["kv_heads"]
        nq, nk = _prompt_lens(case)
        s["cu_q"], s["cu_k"] = _ints(_cum(nq)), _ints(_cum(nk))
        T, Tk = sum(nq), sum(nk)
        if case["ctx"]:
            s["q"] = _randn(g, T, Hq, D, dtype=dtype, std=2.0)
            s["k"], s["v"] = (_randn(g, Tk, H, D, dtype=dtype) for _ in range(2))
        else:  # the three are parts of the rows that one product wrote
            s["q"], s["k"], s["v"] = _randn(g, T, Hq + 2 * H, D, dtype=dtype, std=1.4).split([Hq, H, H], dim=1)
        s["out"] = torch.empty((T, Hq, D), dtype=dtype, device="cuda")
        s["lse"] = torch.empty((T, Hq), device="cuda")
    return s


def _prompt_lens(case):
    nq = _lens(case["B"], case["len"], case["ragged"], least=1)
    ctx = _lens(case["B"], case["ctx"], case["ragged"])
    return nq, [a + b for a, b in zip(nq, ctx)]


# ---------------------------------------------------------------- one pass

def run(s):
    case = s["case"]
    if own:
        return _RUN[case["op"]](s)
    return _PLAIN[case["op"]](s)


def _run_rope(s):
    import paper_2606_10520_amd.unisvq as u
    case = s["case"]
    return u.rope(s["x"], s["pos"], s["table"], interleaved=case["layout"] == "interleaved", inverse=case["inverse"],
                  out=s["out"])


def _run_cache(s):
    import paper_2606_10520_amd.unisvq as u
    cache = (s["k"], s["v"], s["ks"], s["vs"])
    q = u.cache_append(cache, s["table"], s["seq"], s["pos"], s["knew"], s["vnew"], q=s["q"], rope_table=s["rope"],
                       interleaved=s["case"]["layout"] == "interleaved", q_out=s["q_out"])
    k, v = u.cache_read(cache, s["table"], s["start"], s["cu"], s["total"], out=(s["k_out"], s["v_out"]))
    return {"q": q, "k": k, "v": v}


def _run_decode(s):
    import paper_2606_10520_amd.unisvq as u
    out = u.attn_decode(s["q"], (s["k"], s["v"], s["ks"], s["vs"]), s["table"], s["lens"], out=s["out"], lse=s["lse"])
    return {"out": out, "lse": s["lse"]}


def _run_prompt(s):
    import paper_2606_10520_amd.unisvq as u
    out = u.attn_prompt(s["q"], s["k"], s["v"], s["cu_q"], s["cu_k"], causal=s["case"]["causal"], out=s["out"],
                        lse=s["lse"])
    return {"out": out, "lse": s["lse"]}


_RUN = {"rope": _run_rope, "cache": _run_cache, "decode": _run_decode, "prompt": _run_prompt}


def _rotate(x, pos, table, layout, inverse=False):
    """x [T][heads][D] in f32, its first 2 * table.shape[2] dims rotated."""
    half = table.shape[2]
    at = table[pos.long()]
    c, sn = at[:, None, 0], at[:, None, 1]
    if inverse:
        sn = -sn
    if layout == "half":
        a, b = x[..., :half], x[..., half: 2 * half]
        turned = torch.cat([a * c - b * sn, b * c + a * sn], -1)
    else:
        a, b = x[..., 0: 2 * half: 2], x[..., 1: 2 * half: 2]
        turned = torch.stack([a * c - b * sn, b * c + a * sn], -1).flatten(-2)
    return torch.cat([turned, x[..., 2 * half:]], -1)


def _plain_rope(s):
    case = s["case"]
    return _rotate(s["x"].float(), s["pos"], s["table"], case["layout"], case["inverse"]).to(s["x"].dtype)


def _codes(x, top):
    """Scale of each row (the last axis) of x and its codes: -top to top."""
    a = x.abs().amax(-1)
    scale = a / top
    if top == 7:
        scale = scale.to(torch.bfloat16).float()
    scale = torch.where(a < 1e-30, torch.zeros_like(a), scale)
    inv = torch.where(scale > 0, 1 / scale, torch.zeros_like(a))
    code = (x * inv[..., None]).round().clamp(-top, top)
    finite = a < math.inf
    return torch.where(finite, scale, torch.full_like(a, math.nan)), torch.where(finite[..., None], code, torch.zeros_like(x))


def _values(kind, pool, scales):
    """Pool entries as f32 values, scales along the last axis but one."""
    if kind == "i8":
        return pool.float() * scales[..., None]
    if kind == "i4":
        both = torch.stack([pool & 15, pool >> 4], -1).flatten(-2).float() - 8
        return (both.unflatten(-1, (2, -1)) * scales.float()[..., None]).flatten(-2)
    return pool.float()


def _store(kind, pool, scales, at, x):
    """Writes x [T][heads][D], f32, to the pool's places at = (page, token of the page)."""
    if kind == "i8":
        scale, code = _codes(x, 127)
        pool[at[0], :, at[1]] = code.to(torch.int8)
        scales[at[0], :, at[1]] = scale
    elif kind == "i4":
        scale, code = _codes(x.unflatten(-1, (2, -1)), 7)
        code = (code.flatten(-2) + 8).to(torch.uint8).unflatten(-1, (-1, 2))
        pool[at[0], :, at[1]] = code[..., 0] | (code[..., 1] << 4)
        scales[at[0], :, at[1]] = scale.to(torch.bfloat16)
    else:
        pool[at[0], :, at[1]] = x.to(pool.dtype)


def _plain_cache(s):
    case = s["case"]
    kind, page, table = case["kind"], case["page"], s["table"]
    q, k = (_rotate(x.float(), s["pos"], s["rope"], case["layout"]) for x in (s["q"], s["knew"]))
    pos, seq = s["pos"].long(), s["seq"].long()
    at = (table[seq, pos // page].long(), pos % page)
    _store(kind, s["k"], s["ks"], at, k)
    _store(kind, s["v"], s["vs"], at, s["vnew"].float())
    row = torch.arange(s["total"], device="cuda")
    seq = torch.bucketize(row, s["cu"][1:].long(), right=True)
    pos = s["start"][seq] + row - s["cu"][seq]
    at = (table[seq, pos // page].long(), pos % page)
    k, v = (_values(kind, s[n][at[0], :, at[1]], None if s[n + "s"] is None else s[n + "s"][at[0], :, at[1]])
            for n in "kv")
    t = s["qkv"].dtype
    return {"q": q.to(t), "k": k.to(t), "v": v.to(t)}


def _softmax_parts(scores):
    """exp(scores - their largest) in place, the largest (0 where all are masked) and the sums."""
    top = scores.amax(-1, keepdim=True)
    top = torch.where(top == -math.inf, torch.zeros_like(top), top)
    p = scores.sub_(top).exp_()
    return p, top[..., 0], p.sum(-1)


def _plain_decode(s):
    case, q = s["case"], s["q"]
    B, n, Hq, D = q.shape
    H, kind = case["kv_heads"], case["kind"]
    pages = s["table"].clamp(min=0).long()
    width = pages.shape[1] * case["page"]
    pos = torch.arange(width, device="cuda")
    there = (pos < s["lens"][:, None])[:, None, :, None]  # [B][1][width][1]
    k, v = (torch.where(there, _values(kind, s[x][pages], None if s[x + "s"] is None else s[x + "s"][pages])
                        .transpose(1, 2).reshape(B, H, width, D), 0) for x in "kv")
    rows = q.float().reshape(B, n, H, Hq // H, D).permute(0, 2, 3, 1, 4).reshape(B, H, Hq // H * n, D)
    scores = torch.matmul(rows, k.transpose(2, 3).contiguous()) * D ** -0.5
    last = s["lens"][:, None] - n + torch.arange(n, device="cuda")  # the newest position each new token sees
    seen = (pos <= last[..., None]).repeat(1, Hq // H, 1)[:, None]  # [B][1][group * n][width]
    p, top, total = _softmax_parts(torch.where(seen, scores, -math.inf))
    out = torch.matmul(p, v) / torch.where(total > 0, total, 1)[..., None]
    lse = torch.log(total) + top

    def back(x):
        return x.unflatten(2, (Hq // H, n)).movedim(3, 1).flatten(2, 3)
    return {"out": back(out).to(q.dtype), "lse": back(lse)}


def _plain_prompt(s):
    case = s["case"]
    q, k, v = s["q"], s["k"], s["v"]
    T, Hq, D = q.shape
    Tk, H = k.shape[:2]
    at, row = torch.arange(Tk, device="cuda"), torch.arange(T, device="cuda")
    seq_k = torch.bucketize(at, s["cu_k"][1:].long(), right=True)
    seq_q = torch.bucketize(row, s["cu_q"][1:].long(), right=True)
    hidden = seq_q[:, None] != seq_k
    if case["causal"]:  # the last token of a sequence sees all of it
        hidden |= (at - s["cu_k"][1:][seq_k]) > (row - s["cu_q"][1:][seq_q])[:, None]
    rows = q.float().reshape(T, H, Hq // H, D).permute(1, 2, 0, 3).reshape(H, Hq // H * T, D)
    scores = torch.matmul(rows, k.float().permute(1, 2, 0).contiguous()).mul_(D ** -0.5).reshape(Hq, T, Tk)
    p, top, total = _softmax_parts(scores.masked_fill_(hidden, -math.inf))
    out = torch.matmul(p.reshape(H, Hq // H * T, Tk), v.float().transpose(0, 1).contiguous()).reshape(Hq, T, D)
    out /= torch.where(total > 0, total, 1)[..., None]
    return {"out": out.transpose(0, 1).to(q.dtype), "lse": (torch.log(total) + top).T}


_PLAIN = {"rope": _plain_rope, "cache": _plain_cache, "decode": _plain_decode, "prompt": _plain_prompt}


# ---------------------------------------------------------------- what a pass cannot do without

def _entry_bytes(kind, D):
    """Bytes of one token and head in one pool, scales among them."""
    return {"i8": D + 4, "i4": D // 2 + 4}.get(kind, 2 * D)


def work(case):
    D = case["D"]
    if case["op"] == "rope":
        x = case["T"] * case["heads"] * D
        return {"bytes": 4 * x + case["T"] * (4 + 4 * case["rot"]), "flops": 3 * case["T"] * case["heads"] * case["rot"]}
    if case["op"] == "cache":
        T, H = case["B"] * case["new"], case["kv_heads"]
        read = T + (sum(_lens(case["B"], case["ctx"], case["ragged"])) if case["read_all"] else 0)
        entry = _entry_bytes(case["kind"], D)
        return {"bytes": T * (4 * case["q_heads"] * D + 4 * H * D + 2 * H * entry + 4 * case["rot"] + 8)
                + read * 2 * H * (entry + 2 * D),
                "flops": 3 * T * (case["q_heads"] + H) * case["rot"] + 4 * T * H * D + 2 * read * H * D}
    if case["op"] == "decode":
        lens = _lens(case["B"], case["len"], case["ragged"])
        rows = case["B"] * case["q_len"] * case["q_heads"]
        pairs = sum(max(0, n - j) for n in lens for j in range(case["q_len"])) * case["q_heads"]
        return {"bytes": sum(lens) * 2 * case["kv_heads"] * _entry_bytes(case["kind"], D) + rows * (4 * D + 4),
                "flops": 4 * D * pairs}
    nq, nk = _prompt_lens(case)
    pairs = sum(a * b - (a * (a - 1) // 2 if case["causal"] else 0) for a, b in zip(nq, nk)) * case["q_heads"]
    return {"bytes": sum(nq) * case["q_heads"] * (4 * D + 4) + sum(nk) * case["kv_heads"] * 4 * D,
            "flops": 4 * D * pairs}


# ---------------------------------------------------------------- the same from the definition, in 64 bits

def _turn64(x, pos, table, layout, sign=1.0):
    """Each pair as a complex number times cos + i sin."""
    y, half = x.double().clone(), table.shape[2]
    t = table.double()[pos.long()]
    w = torch.complex(t[:, 0], sign * t[:, 1])[:, None]
    first, second = (slice(0, half), slice(half, 2 * half)) if layout == "half" else (slice(0, 2 * half, 2), slice(1, 2 * half, 2))
    z = torch.complex(y[..., first], y[..., second]) * w
    y[..., first], y[..., second] = z.real, z.imag
    return y


def _stored64(kind, x, dtype):
    """The values that a cache holds for x, in 64 bits."""
    if kind not in ("i8", "i4"):
        return x.to(DTYPE[kind]).double()
    parts, top = (1, 127) if kind == "i8" else (2, 7)
    x = x.unflatten(-1, (parts, -1))
    scale = x.abs().amax(-1, keepdim=True) / top
    scale = scale.to(torch.bfloat16 if kind == "i4" else torch.float32).double()
    code = torch.clamp(torch.round(x / scale), -top, top)
    return torch.where(scale > 0, code * scale, torch.zeros_like(code)).flatten(-2)


def _held64(s, kind, b, n):
    """Keys and values [n][heads][D] of the first n tokens of sequence b, in 64 bits."""
    out = []
    for name in "kv":
        pool, scales, rows = s[name], s[name + "s"], []
        for i in range(-(-n // pool.shape[2])):
            page = int(s["table"][b, i])
            x = pool[page]
            if kind == "i8":
                x = x.double() * scales[page].double()[..., None]
            elif kind == "i4":
                lo, hi = (x % 16).double() - 8, (x // 16).double() - 8
                wide = torch.empty((*x.shape[:2], 2 * x.shape[2]), dtype=torch.float64, device="cuda")
                wide[..., 0::2], wide[..., 1::2] = lo, hi
                x = wide * scales[page].double().repeat_interleave(x.shape[2], -1)
            rows.append(x.double().transpose(0, 1))
        out.append(torch.cat(rows)[:n] if rows else torch.zeros((0, pool.shape[1], s["q"].shape[-1]), dtype=torch.float64, device="cuda"))
    return out


def _attend64(q, k, v, last):
    """q [n][Hq][D], k, v [m][H][D] in 64 bits; row i sees positions up to last[i]."""
    n, Hq, D = q.shape
    m, H = k.shape[:2]
    out = torch.zeros((n, Hq, D), dtype=torch.float64, device="cuda")
    lse = torch.full((n, Hq), -math.inf, dtype=torch.float64, device="cuda")
    if m == 0 or n == 0:
        return out, lse
    hide = torch.arange(m, device="cuda")[None, :] > last[:, None]
    some = ~hide.all(1)
    for h in range(Hq):
        z = (q[:, h] @ k[:, h * H // Hq].T.contiguous()) / math.sqrt(D)
        z[hide] = -math.inf
        lse[:, h] = torch.logsumexp(z, 1)
        w = torch.softmax(z, 1)
        w[~some] = 0
        out[:, h] = w @ v[:, h * H // Hq].contiguous()
    return out, lse


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "rope":
        return _turn64(s["x"], s["pos"], s["table"], case["layout"], -1.0 if case["inverse"] else 1.0)
    if case["op"] == "cache":
        B, new, kind = case["B"], case["new"], case["kind"]
        before = _lens(B, case["ctx"], case["ragged"])
        fresh = {"k": _stored64(kind, _turn64(s["knew"], s["pos"], s["rope"], case["layout"]), case["dtype"]),
                 "v": _stored64(kind, s["vnew"].double(), case["dtype"])}
        got = {"k": [], "v": []}
        for b in range(B):
            old = _held64(s, kind, b, before[b]) if case["read_all"] else None
            for i, name in enumerate("kv"):
                part = fresh[name][b * new: (b + 1) * new]
                got[name].append(torch.cat([old[i], part]) if case["read_all"] else part)
        return {"q": _turn64(s["q"], s["pos"], s["rope"], case["layout"]), "k": torch.cat(got["k"]), "v": torch.cat(got["v"])}
    out, lse = [], []
    if case["op"] == "decode":
        n = case["q_len"]
        for b, m in enumerate(_lens(case["B"], case["len"], case["ragged"])):
            k, v = _held64(s, case["kind"], b, m)
            o, z = _attend64(s["q"][b].double(), k, v, torch.arange(n, device="cuda") + m - n)
            out.append(o)
            lse.append(z)
        return {"out": torch.stack(out), "lse": torch.stack(lse)}
    nq, nk = _prompt_lens(case)
    cq, ck = _cum(nq), _cum(nk)
    for b in range(case["B"]):
        q = s["q"][cq[b]: cq[b + 1]].double()
        k, v = (s[x][ck[b]: ck[b + 1]].double() for x in "kv")
        last = torch.arange(nq[b], device="cuda") + (nk[b] - nq[b]) if case["causal"] else torch.full((nq[b],), nk[b], device="cuda")
        o, z = _attend64(q, k, v, last)
        out.append(o)
        lse.append(z)
    return {"out": torch.cat(out), "lse": torch.cat(lse)}
