"""Attention over the paged cache against a plain 64-bit implementation on the values that the cache holds."""
import numpy as np
import pytest

import attn_ref as ref
from test_gpu_cache import DEV, DT, ints, page_table

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def u():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2606_10520_amd.unisvq as u
    u.load()
    return u


def filled(u, kind, lens, page, H, D, seed, spare=1, spread=1.0):
    """A cache with random contents of these lengths, everything past them NaN or garbage; its page table; and the
    values it holds, fp64 [sequence] of [len][H][D]."""
    rng = np.random.default_rng(seed)
    t, pages = page_table(lens, page, seed, spare)
    used = np.zeros((pages, page), dtype=bool)
    for b, n in enumerate(lens):
        for p in range(n):
            used[t[b, p // page], p % page] = True
    free = torch.from_numpy(~used[:, None, :].repeat(H, 1))
    x = rng.standard_normal((2, pages, H, page, D)).astype(np.float32) * np.exp2(rng.uniform(-spread, spread, (2, pages, H, page, 1))).astype(np.float32)
    if kind in ("f16", "bf16"):
        pools = [torch.from_numpy(p).to(DT[kind]) for p in x]
        values = [p.double().numpy() for p in pools]
        for p in pools:
            p[free] = float("nan")
        cache = (*[p.to(DEV) for p in pools], None, None)
    else:
        pools, scales, values = [], [], []
        for p in x:
            code, scale = ref.quantise(p, kind)
            values.append(ref.dequantise(code, scale, kind).astype(np.float64))
            if kind == "i4":
                n = (code + 8).astype(np.uint8)
                pools.append(torch.from_numpy(n[..., 0::2] | n[..., 1::2] << 4))
                scales.append(torch.from_numpy(scale).bfloat16())
            else:
                pools.append(torch.from_numpy(code))
                scales.append(torch.from_numpy(scale))
            scales[-1][free] = float("nan")
        cache = (*[p.to(DEV) for p in pools], *[s.to(DEV) for s in scales])
    held = []
    for b, n in enumerate(lens):
        at = [(t[b, p // page], p % page) for p in range(n)]
        held.append([np.stack([v[i, :, j] for i, j in at]) if n else np.zeros((0, H, D)) for v in values])
    return cache, torch.from_numpy(t).to(DEV), held


def run_and_check(u, cache, pt, held, lens, q, kind, dtype, scale=None, **more):
    B, n, HQ, D = q.shape
    lse = torch.full((B, n, HQ), 7.0, device=DEV)
    out = u.attn_decode(q.to(DEV), cache, pt, ints(lens), scale=scale, lse=lse, **more)
    weights = "bf16" if kind == "bf16" else "f16"
    worst = 0.0
    for b in range(B):
        k, v = held[b]
        r = ref.attention(q[b].double().numpy(), k, v, np.arange(n) + lens[b] - n, scale or D ** -0.5)
        vmax = np.abs(v).max() if v.size else 0.0
        worst = max(worst, ref.check(out[b].double().cpu().numpy(), lse[b].double().cpu().numpy(), r, max(1, lens[b]), weights, dtype, vmax))
    return out, lse, worst


KINDS = [("i8", "f16"), ("i8", "bf16"), ("i4", "f16"), ("i4", "bf16"), ("f16", "f16"), ("bf16", "bf16")]
LENS = [0, 1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 129, 200, 257, 513]


@pytest.mark.parametrize("kind,dtype", KINDS)
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("H,group,q_len", [(1, 1, 1), (2, 4, 1), (2, 1, 3), (1, 5, 4), (2, 8, 4), (1, 3, 16)])
def test_lengths(u, kind, dtype, D, H, group, q_len):
    page = {1: 16, 2: 64}[H]
    cache, pt, held = filled(u, kind, LENS, page, H, D, seed=D + group)
    q = (torch.randn((len(LENS), q_len, H * group, D), generator=torch.Generator().manual_seed(1)) * 2).to(DT[dtype])
    run_and_check(u, cache, pt, held, LENS, q, kind, dtype)


@pytest.mark.parametrize("kind,dtype", KINDS)
@pytest.mark.parametrize("page", [16, 32, 64, 128, 256])
def test_one_long_sequence(u, kind, dtype, page):
    """A length that is split over many workgroups and joined."""
    lens = [5003]
    cache, pt, held = filled(u, kind, lens, page, 2, 128, seed=page, spare=3)
    q = (torch.randn((1, 1, 8, 128), generator=torch.Generator().manual_seed(2)) * 3).to(DT[dtype])
    assert u.attn_decode_workspace_bytes(1, 1, 8, 2, 128, 5003) > 0
    first, lse, _ = run_and_check(u, cache, pt, held, lens, q, kind, dtype)
    again, lse2, _ = run_and_check(u, cache, pt, held, lens, q, kind, dtype)
    assert torch.equal(first, again) and torch.equal(lse, lse2)
    # other splits: what the lengths are said to be at most, too little included
    for most in (1, 100, 1000, 6000):
        run_and_check(u, cache, pt, held, lens, q, kind, dtype, max_len=most)


@pytest.mark.parametrize("kind,dtype", KINDS)
def test_scores_and_scales_far_apart(u, kind, dtype):
    """Scores up to hundreds (one key takes all the weight, wherever it is), values' scales over a factor of 2^24."""
    lens = [300, 77]
    cache, pt, held = filled(u, kind, lens, 32, 2, 128, seed=9, spread=3.0 if kind == "f16" else 12.0)
    q = (torch.randn((2, 2, 4, 128), generator=torch.Generator().manual_seed(3)) * 10).to(DT[dtype])
    run_and_check(u, cache, pt, held, lens, q, kind, dtype, scale=0.05 if kind != "f16" else None)


def test_queries_of_all_magnitudes_on_codes(u):
    """bf16 queries beyond fp16's range, and rows of zeros."""
    lens = [90, 90, 90]
    cache, pt, held = filled(u, "i8", lens, 16, 1, 128, seed=4)
    q = torch.randn((3, 1, 2, 128), generator=torch.Generator().manual_seed(4)).bfloat16()
    q[0] *= 1e30
    q[1] *= 1e-30
    q[2, 0, 1] = 0
    for b, scale in ((0, 1e-30), (1, 1e28), (2, 0.1)):
        run_and_check(u, cache, pt[b:b + 1].contiguous(), held[b:b + 1], lens[b:b + 1], q[b:b + 1], "i8", "bf16", scale=scale)


@pytest.mark.parametrize("kind", ["i8", "f16"])
def test_pages_that_are_missing(u, kind):
    """Places without a page are as if they were not there."""
    lens, page, H, D = [100], 16, 1, 64
    cache, pt, held = filled(u, kind, lens, page, H, D, seed=6)
    gone = [1, 4, 6]  # of the pages of the sequence
    pt[0, gone[0]], pt[0, gone[1]], pt[0, gone[2]] = -1, 10 ** 9, cache[0].shape[0]
    keep = np.array([p for p in range(100) if p // page not in gone])
    k, v = (x[keep] for x in held[0])
    q = torch.randn((1, 2, 2, D)).half()
    lse = torch.empty((1, 2, 2), device=DEV)
    out = u.attn_decode(q.to(DEV), cache, pt, ints(lens), lse=lse)
    last = [int(np.searchsorted(keep, p, side="right")) - 1 for p in (98, 99)]
    ref.check(out[0].double().cpu().numpy(), lse[0].double().cpu().numpy(), ref.attention(q[0].double().numpy(), k, v, last, D ** -0.5),
              100, "f16", "f16", np.abs(v).max())
    pt.fill_(-1)
    out = u.attn_decode(q.to(DEV), cache, pt, ints(lens), lse=lse)
    assert not out.any() and torch.isneginf(lse).all()


def test_more_heads_than_workgroups(u):
    lens = [300, 1, 0, 129]
    cache, pt, held = filled(u, "i8", lens, 16, 520, 64, 41)
    q = torch.from_numpy(np.random.default_rng(42).standard_normal((4, 1, 520, 64))).half()
    run_and_check(u, cache, pt, held, lens, q, "i8", "f16")


@pytest.mark.parametrize("kind,D,H", [("i4", 64, 25), ("f16", 64, 25), ("f16", 128, 25), ("i8", 128, 50), ("f16", 64, 50),
                                      ("i4", 64, 100), ("f16", 64, 100), ("i8", 64, 150), ("f16", 64, 150)])
@pytest.mark.parametrize("longest,max_len", [(1024, 0), (1025, 0), (1000, 300), (129, 0)])
def test_from_few_items_to_many(u, kind, D, H, longest, max_len):
    """Whole items with four or eight wavefronts, and shares of them: both sides of what chooses between them."""
    lens = [longest, 300 % longest, 0, 1]
    cache, pt, held = filled(u, kind, lens, 32, H, D, 51)
    q = torch.from_numpy(np.random.default_rng(52).standard_normal((4, 1, H, D))).half()
    run_and_check(u, cache, pt, held, lens, q, kind, "f16", max_len=max_len)


@pytest.mark.parametrize("H,lens", [
    (8, [7000, 2300, 1, 4097]),  # rounded up to whole shares
    (8, [31 * i % 2000 for i in range(60)]),  # too many items for that
    (3, [130] * 70 + [9000, 0]),  # more sequences than a wavefront has lanes, some as long as many
])
def test_ragged_batches(u, H, lens):
    cache, pt, held = filled(u, "i8", lens, 64, H, 64, 61)
    q = torch.from_numpy(np.random.default_rng(62).standard_normal((len(lens), 1, 2 * H, 64))).half()
    run_and_check(u, cache, pt, held, lens, q, "i8", "f16")


def test_lengths_beyond_the_page_table_and_below_zero(u):
    cache, pt, held = filled(u, "i8", [64, 64], 16, 1, 128, seed=8)
    q = torch.randn((2, 1, 4, 128)).half()
    want, lse, _ = run_and_check(u, cache, pt, held, [64, 64], q, "i8", "f16")
    out = u.attn_decode(q.to(DEV), cache, pt, ints([2 ** 31 - 1, -5]))
    assert torch.equal(out[0], want[0]) and not out[1].any()


def test_strides_of_queries_and_outputs(u):
    cache, pt, held = filled(u, "i8", [50, 20], 16, 2, 128, seed=12)
    q = torch.randn((2, 8, 128)).half()
    want = u.attn_decode(q.to(DEV), cache, pt, ints([50, 20]))
    wide = torch.zeros((2, 12, 128), dtype=torch.float16, device=DEV)
    wide[:, 2:10] = q.to(DEV)
    out = torch.full((2, 12, 128), 3.0, dtype=torch.float16, device=DEV)
    got = u.attn_decode(wide[:, 2:10], cache, pt, ints([50, 20]), out=out[:, 1:9])
    assert torch.equal(got, want) and (out[:, 0] == 3).all() and (out[:, 9:] == 3).all()


@pytest.mark.parametrize("kind,dtype", KINDS)
def test_not_a_number_where_it_is_seen_only(u, kind, dtype):
    """A value that is not finite reaches the rows that see it and no others."""
    cache, pt, held = filled(u, kind, [70, 70], 16, 1, 64, seed=13)
    q = torch.randn((2, 4, 1, 64)).to(DT[dtype])
    want = u.attn_decode(q.to(DEV), cache, pt, ints([70, 70])).cpu()
    for at in (69, 67):  # seen by the last row, and by the last three
        page = int(pt[0, at // 16])
        pool = cache[1] if kind in ("f16", "bf16") else cache[3]
        for bad in (float("nan"), float("inf")):
            was = pool[page, 0, at % 16].clone()
            if kind == "i8":
                pool[page, 0, at % 16] = bad
            else:  # one value, or the scale of one half
                pool[page, 0, at % 16, 0] = bad
            out = u.attn_decode(q.to(DEV), cache, pt, ints([70, 70])).cpu()
            assert torch.equal(out[1], want[1]) and torch.equal(out[0, :at - 66], want[0, :at - 66])
            assert (~torch.isfinite(out[0, at - 66:])).any(-1).all()
            pool[page, 0, at % 16] = was


def test_graph_replays_follow_lengths_and_contents(u):
    """A decoding step (write a token, attend) recorded once and replayed as the sequences grow, eager work between."""
    H, G, D, B, page = 2, 4, 128, 3, 16
    start = [5, 40, 15]
    steps = 4
    _, pages = page_table([n + steps for n in start], page, 1)
    t, pages = page_table([n + steps for n in start], page, 1)
    pt = torch.from_numpy(t).to(DEV)
    cache = u.new_cache(pages, H, page, D, "i8")
    gen = torch.Generator(device=DEV).manual_seed(0)
    rnd = lambda *s: torch.randn(s, generator=gen, device=DEV).half()
    seqs, pos = np.repeat(np.arange(B), start), np.concatenate([np.arange(n) for n in start])
    old = rnd(2, sum(start), H, D)
    table = u.rope_table(64, D)
    u.cache_append(cache, pt, ints(seqs), ints(pos), old[0], old[1], rope_table=table)
    q, k, v = rnd(B, H * G, D), rnd(B, H, D), rnd(B, H, D)
    qr, out = torch.empty_like(q), torch.empty_like(q)
    lens, where = ints(start), ints(start)
    ws = torch.empty(max(16, u.attn_decode_workspace_bytes(B, 1, H * G, H, D, t.shape[1] * page)), dtype=torch.uint8, device=DEV)

    def step():
        u.cache_append(cache, pt, None, where, k, v, q=q, rope_table=table, q_out=qr)
        u.attn_decode(qr, cache, pt, lens, out=out, workspace=ws)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        lens += 1
        step()
    torch.cuda.current_stream().wait_stream(side)
    lens -= 1
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for n in range(steps):
        for x in (q, k, v):
            x.copy_(rnd(*x.shape))
        lens += 1
        out.fill_(9)
        graph.replay()
        torch.cuda.synchronize()
        got = out.clone()
        before = [c.clone() for c in cache]
        step()
        torch.cuda.synchronize()
        assert torch.equal(got, out) and all(torch.equal(a, b) for a, b in zip(before, cache))
        where += 1


def test_another_stream(u):
    cache, pt, held = filled(u, "i8", [3000], 64, 2, 128, seed=15)
    q = torch.randn((1, 8, 128), device=DEV).half()
    want = u.attn_decode(q, cache, pt, ints([3000]))
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    lens = ints([3000])
    torch.cuda.synchronize()
    got = u.attn_decode(q, cache, pt, lens, stream=s)
    s.synchronize()
    assert torch.equal(got, want)


def test_cache_past_four_gib(u):
    """Entries whose byte offsets pass 32 bits."""
    D, H, page = 128, 8, 256
    pages = (1 << 32) // (H * page * D) + 5
    cache = tuple(torch.empty((pages, H, page) + ((D,) if i < 2 else ()), dtype=torch.int8 if i < 2 else torch.float32, device=DEV)
                  for i in range(4))
    small, pt0, held = filled(u, "i8", [700], page, H, D, seed=16, spare=0)
    at = [pages - 1, 0, pages - 3]
    for i, p in enumerate(pt0[0].tolist()):
        for a, b in zip(cache, small):
            a[at[i]] = b[p]
    q = torch.randn((1, 1, 8, 128)).half()
    run_and_check(u, cache, ints([at]), held, [700], q, "i8", "f16")
