"""Shared prefixes, entry weights and eviction on the GPU against plain 64-bit
forms (tests/shared_ref.py, which derives the bounds)."""
import numpy as np
import pytest
import torch

import shared_ref as ref
from draft_ref import HALF, f64
from gpu_case import guarded
from paper_2607_06827_amd import inputs
from paper_2607_06827_amd import speechkv as skv
from test_gpu_draft import i32, make_cache

pytestmark = [pytest.mark.gpu,
              pytest.mark.skipif(not torch.cuda.is_available(), reason="needs a GPU")]

DEV = "cuda"
BF, F32 = torch.bfloat16, torch.float32


def check(got, want, bound, what):
    got = f64(got)
    same = (got == want) | (np.isnan(got) & np.isnan(want))
    off = np.where(same, -1.0, np.abs(np.where(same, 0.0, got) - np.where(same, 0.0, want)) - bound)
    assert np.all(off <= 0), (what, np.max(off), np.unravel_index(np.argmax(off), off.shape))


def poison(cache, lens):
    """NaN in every row of the pools that no entry of the cache has."""
    used = torch.zeros(cache.k_pages.shape[0], cache.k_pages.shape[2], dtype=torch.bool, device=DEV)
    ps, pages = cache.k_pages.shape[2], cache.k_pages.shape[0]
    for b, n in enumerate(lens):
        s = torch.arange(n, device=DEV)
        page = cache.block_table[b, s // ps].long()
        ok = (page >= 0) & (page < pages)
        used[page[ok], (s % ps)[ok]] = True
    for x in (cache.k_pages, cache.v_pages):
        x[~used[:, None].expand(-1, x.shape[1], -1)] = float("nan")


# ------------------------------------------------------------ shared prefixes

SHARED = [
    # dtype, D, Hq, Hkv, page, prefix lengths, group_start, own lengths, splits
    (BF, 128, 16, 8, 16, [126], [0, 8], [40] * 8, 0),
    (BF, 128, 4, 2, 16, [0, 1, 33, 64], [0, 1, 3, 3, 6], [5, 0, 1, 32, 33, 64], 0),
    (BF, 64, 8, 8, 8, [500], [0, 20], [i % 4 for i in range(20)], 3),
    (BF, 128, 64, 8, 64, [1000, 31, 700], [0, 9, 9, 12], [100 + i for i in range(12)], 7),
    (F32, 64, 16, 4, 16, [217, 90], [0, 5, 7], [33, 1, 0, 9, 20, 3, 31], 0),
    (F32, 128, 2, 1, 32, [65], [0, 3], [0, 0, 0], 2),
    (BF, 128, 2, 2, 256, [2000], [0, 70], [3] * 70, 0),
    (BF, 64, 16, 2, 16, [0], [0, 4], [0, 5, 0, 70], 4),
    (BF, 128, 8, 1, 128, [3000], [2, 5], [300, 20, 0, 1, 2, 900, 77], 0),  # sequences of no group
    (F32, 64, 8, 2, 16, [40, 41, 0, 300], [0, 0, 2, 2, 3], [7, 0, 5, 100], 1024),
    (BF, 128, 16, 2, 16, [7532], [0, 3], [5, 1000, 0], 0),
    (BF, 64, 1, 1, 8, [5], [0, 1], [0], 0),
]


class Shared:
    def __init__(self, case, seed=0):
        (self.dt, self.D, self.Hq, self.Hkv, page, self.prefix, self.start, self.own, self.splits) = SHARED[case]
        self.B = len(self.own)
        self.pc = make_cache(len(self.prefix), max(self.prefix + [1]), self.Hkv, self.D, self.dt, page, seed=400 + case + seed)
        self.oc = make_cache(self.B, max(self.own + [1]), self.Hkv, self.D, self.dt, page, seed=500 + case + seed)
        poison(self.pc, self.prefix)
        poison(self.oc, self.own)
        self.q = inputs.normal((self.B, self.Hq, self.D), 600 + case + seed, dtype=self.dt).to(DEV)
        self.most = max(1, max(e - s for s, e in zip(self.start, self.start[1:])))

    def run(self, splits=None, stream=None, out=None, lse=None, ws=None, slack=0):
        splits = self.splits if splits is None else splits
        bound = [min(max(x) + slack, c.block_table.shape[1] * c.k_pages.shape[2])
                 for x, c in ((self.prefix, self.pc), (self.own, self.oc))]
        n, m = len(self.prefix), min(self.B, self.most + slack)
        need = skv.speechkv_shared_workspace_bytes(self.B, n, m, self.Hq, self.Hkv, self.D, *bound, splits)
        guards = []
        if out is None:
            (out, g1), (lse, g2), (ws, g3) = (guarded((self.B, self.Hq, self.D), self.dt, DEV),
                                              guarded((self.B, self.Hq), F32, DEV), guarded((need // 4,), F32, DEV))
            guards = [g1, g2, g3]
        skv.speechkv_shared_attn(self.q, self.pc, i32(self.prefix), bound[0], i32(self.start), m, self.oc,
                                 i32(self.own), bound[1], out, lse=lse, num_splits=splits, workspace=ws, stream=stream)
        torch.cuda.synchronize()
        for g in guards:
            g("shared")
        return out, lse

    def check(self, out, lse, what, parts=1088):
        pk, pv, ok, ov = (f64(x) for x in (self.pc.k_pages, self.pc.v_pages, self.oc.k_pages, self.oc.v_pages))
        pt, ot, q = f64(self.pc.block_table).astype(int), f64(self.oc.block_table).astype(int), f64(self.q)
        for b in range(self.B):
            sources = [ref.entries(ok, ov, ot, b, self.own[b])[1:]]
            for j, (s, e) in enumerate(zip(self.start, self.start[1:])):
                if s <= b < e:
                    sources.append(ref.entries(pk, pv, pt, j, self.prefix[j])[1:])
            o, bound, l, lbound = ref.attention(q[b], sources, self.D ** -0.5, HALF[self.dt], parts)
            check(out[b], o, bound, (what, b))
            check(lse[b], l, lbound, (what, "lse", b))


@pytest.mark.parametrize("case", range(len(SHARED)))
def test_shared(case):
    x = Shared(case)
    out, lse = x.run()
    x.check(out, lse, case)
    again, lse2 = x.run()
    assert torch.equal(out, again) and torch.equal(lse, lse2)
    loose, lse3 = x.run(slack=300)  # host bounds beyond the real sizes
    x.check(loose, lse3, "loose")


@pytest.mark.parametrize("splits", [1, 2, 5, 33])
def test_shared_splits(splits):
    x = Shared(3)
    x.check(*x.run(splits), splits)


def test_shared_missing_pages_and_bad_lengths():
    """Entries without a page are not there; lengths beyond the bounds or below 0
    are cut; group starts out of range are cut."""
    x = Shared(1)
    x.prefix, x.own = [60, 64, 50, 64], [64, 48, 10, 64, 33, 64]
    x.pc.k_pages.normal_()
    x.pc.v_pages.normal_()
    x.oc.k_pages.normal_()
    x.oc.v_pages.normal_()
    x.pc.block_table[1, 2] = -1
    x.pc.block_table[3, 0] = 10 ** 6
    x.oc.block_table[3] = -7
    x.oc.block_table[4, 1] = x.oc.k_pages.shape[0]
    out, lse = x.run()
    x.check(out, lse, "missing")
    out2, lse2 = torch.empty_like(out), torch.empty_like(lse)
    need = skv.speechkv_shared_workspace_bytes(6, 4, 3, 4, 2, 128, 64, 64)
    skv.speechkv_shared_attn(x.q, x.pc, i32([60, 64, 50, 2 ** 31 - 1]), 64, i32([-5, 1, 3, 3, 99]), 3, x.oc,
                             i32([99, 48, 10, 2 ** 30, 33, 64]), 64, out2, lse=lse2,
                             workspace=torch.empty(need, dtype=torch.uint8, device=DEV))
    x.check(out2, lse2, "cut")
    x.own = [0] * 6
    x.start = [0] * 5
    x.check(*x.run(), "nothing to see")


@pytest.mark.parametrize("dt", [BF, F32])
def test_shared_values_that_are_not_finite(dt):
    """An infinite value reaches the rows that see it, in its own element, and no
    others; the last entry's too, though its tile ends behind it."""
    for where in ("prefix", "own"):
        x = Shared(0 if dt == BF else 4)
        c, b = (x.pc, 0) if where == "prefix" else (x.oc, 0)
        n = x.prefix[0] if where == "prefix" else x.own[0]
        page = int(c.block_table[b, (n - 1) // 16])
        c.v_pages[page, 0, (n - 1) % 16, 7] = float("inf")
        out, lse = x.run()
        members = range(x.start[0], x.start[1]) if where == "prefix" else [0]
        G = x.Hq // x.Hkv
        hit = torch.zeros_like(out, dtype=torch.bool)
        for m in members:
            hit[m, :G, 7] = True
        assert bool(torch.isposinf(out[hit]).all()) and bool(torch.isfinite(out[~hit]).all())
        assert bool(torch.isfinite(lse).all())


def test_shared_is_attention_over_the_whole():
    """A group of one with its prefix and own entries in one cache is a decoding
    step over that cache."""
    x = Shared(10)
    b = 1
    n, m = x.prefix[0], x.own[b]
    whole = make_cache(1, n + m, x.Hkv, x.D, x.dt, 16)
    s = torch.arange(n + m, device=DEV)
    for name in ("k_pages", "v_pages"):
        rows = []
        for c, row, L in ((x.pc, 0, n), (x.oc, b, m)):
            i = torch.arange(L, device=DEV)
            rows.append(getattr(c, name)[c.block_table[row, i // 16].long(), :, i % 16])
        getattr(whole, name)[whole.block_table[0, s // 16].long(), :, s % 16] = torch.cat(rows)
    want = torch.empty_like(x.q[:1])
    skv.speechkv_decode_attn(x.q[b:b + 1], whole, i32([n + m]), n + m, want, num_splits=1)
    out, _ = x.run()
    assert float((out[b].float() - want[0].float()).abs().max()) <= 3 * 2.0 ** -8 * float(want.abs().max())


def test_shared_captured_and_on_another_stream():
    x, y = Shared(3), Shared(3, seed=50)
    bound = max(x.prefix), max(x.own)
    need = skv.speechkv_shared_workspace_bytes(x.B, 3, x.most, x.Hq, x.Hkv, x.D, *bound)
    fresh = lambda: (torch.zeros_like(x.q), torch.zeros((x.B, x.Hq), device=DEV),  # noqa: E731
                     torch.empty(need, dtype=torch.uint8, device=DEV))
    lens = [i32(x.prefix), i32(x.start), i32(x.own)]

    def step(o, stream=None):
        skv.speechkv_shared_attn(x.q, x.pc, lens[0], bound[0], lens[1], x.most, x.oc, lens[2], bound[1], o[0], lse=o[1],
                                 workspace=o[2], stream=stream)

    got = fresh()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(got)
    side = torch.cuda.Stream()
    # (pools come with their tables: what no entry uses is NaN)
    tensors = lambda s: (s.q, s.pc.k_pages, s.pc.v_pages, s.pc.block_table, s.oc.k_pages, s.oc.v_pages,  # noqa: E731
                         s.oc.block_table)
    keep = [t.clone() for t in tensors(x)]
    for new in (tensors(y), keep, (y.q, *keep[1:])):
        for a, b in zip(tensors(x), new):
            a.copy_(b)
        want = fresh()
        torch.cuda.synchronize()
        step(want, stream=side)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


# -------------------------------------------------------------- entry weights

WEIGHTS = [
    # dtype, D, Hq, Hkv, page, lengths, rows, how rows see: "last", "all", "prompt", "any"
    (BF, 128, 16, 8, 16, [166], 1, "last"),
    (BF, 128, 16, 8, 16, [5, 64, 65, 0, 300], 1, "last"),
    (BF, 64, 8, 1, 8, [700, 1, 33], 4, "last"),
    (BF, 128, 4, 2, 64, [100, 40], 200, "any"),
    (BF, 128, 2, 2, 16, [90, 17, 0], 33, "any"),
    (F32, 64, 16, 4, 16, [217, 90], 1, "all"),
    (F32, 128, 4, 4, 32, [130], 70, "any"),
    (BF, 64, 64, 8, 128, [500], 17, "last"),
    (F32, 128, 8, 1, 256, [1000, 999], 2, "last"),
    (BF, 128, 2, 1, 16, [7, 3], 300, "last"),  # rows that see nothing
    (BF, 64, 8, 8, 16, [9000, 4001, 17], 1, "last"),  # several steps of keys a wave
    (BF, 64, 8, 1, 16, [90], 1100, "any"),  # more row tiles than are looked through at once
    (F32, 128, 8, 1, 16, [70], 1030, "last"),
    # two stretches of keys a block: one, two and more of them in a sequence, odd and even
    (BF, 128, 8, 8, 16, [130, 64, 65, 0, 192, 193, 256, 257, 1, 70, 120], 37, "any"),
    (BF, 64, 32, 32, 8, [300, 129, 63], 40, "last"),
    (F32, 128, 16, 16, 32, [100, 33, 32, 161, 7], 35, "any"),
    (F32, 64, 64, 32, 16, [310, 1, 128], 20, "last"),
    (BF, 128, 16, 16, 16, [500, 449, 385, 70], 35, "last"),
    (BF, 128, 32, 16, 64, [450, 65, 512, 1], 18, "any"),
    (F32, 64, 32, 32, 16, [510, 300], 36, "any"),
]


@pytest.mark.parametrize("case", range(len(WEIGHTS)))
@pytest.mark.parametrize("form", ["add", "in place", "from zero"])
def test_weights(case, form):
    dt, D, Hq, Hkv, page, lens, n, how = WEIGHTS[case]
    B, most, G = len(lens), max(lens), Hq // Hkv
    cache = make_cache(B, most, Hkv, D, dt, page, seed=700 + case)
    poison(cache, lens)
    # rows of a wider tensor, heads outermost in the lse
    q = inputs.normal((B, n + 3, Hq + 1, D), 800 + case, dtype=dt).to(DEV)[:, 2:n + 2, 1:]
    rng = np.random.default_rng(case)
    seen = np.array([[L - (n - 1 - i) for i in range(n)] if how == "last" else [L] * n if how == "all" else
                     rng.integers(-2, L + 3, n) for L in lens])
    scale = D ** -0.5
    K, t = f64(cache.k_pages), f64(cache.block_table).astype(int)
    lse = np.full((B, Hq, n), -np.inf)
    q64 = f64(q)
    parts = []
    for b, L in enumerate(lens):
        keys = ref.entries(K, K, t, b, L)[1]
        parts.append(keys)
        for h in range(Hq):
            z = scale * (q64[b, :, h] @ keys[:, h // G].T)
            for i in range(n):
                s = min(max(seen[b, i], 0), L)
                if s:
                    lse[b, h, i] = np.log(np.exp(z[i, :s] - z[i, :s].max()).sum()) + z[i, :s].max()
    capacity = most + 5
    lse_t = torch.tensor(lse.transpose(1, 0, 2).copy(), dtype=F32, device=DEV).transpose(0, 1)
    had = torch.rand(B, Hkv, capacity, device=DEV)
    out, guard = guarded((B, Hkv, capacity), F32, DEV, fill=-3.0)
    before = None if form == "from zero" else had
    if form == "in place":
        out.copy_(had)
        before = out
    visible = None if how == "last" else i32(seen.tolist())
    skv.speechkv_attn_weights(q, lse_t, cache, i32(lens), min(most + 5, cache.block_table.shape[1] * page), out,
                              weights=before, visible=visible)
    torch.cuda.synchronize()
    guard("weights")
    lse32 = f64(lse_t)
    for b, L in enumerate(lens):
        assert bool((out[b, :, L:] == (had[b, :, L:] if form == "in place" else -3.0)).all())
        for g in range(Hkv):
            start = f64(had[b, g, :L]) if form != "from zero" else np.zeros(L)
            rows = q64[b, :, g * G:(g + 1) * G].reshape(n * G, D)
            l = lse32[b, g * G:(g + 1) * G].T.reshape(n * G)
            want, bound = ref.gathered(rows, l, np.repeat(np.clip(seen[b], 0, L), G), parts[b][:, g], scale, start)
            check(out[b, g, :L], want, bound, (case, b, g))


def test_weights_of_a_row_add_up_to_one():
    """Prompt rows with speechkv_prefill_attn's lse: each row that sees anything
    gives its heads' weights, one in all, and none to entries it does not see."""
    B, P, T, N, w, Hq, Hkv, D = 2, 5, 31, 7, 4, 4, 2, 128
    rows, L = P + T + N, P + 8 + N
    cache = make_cache(B, L, Hkv, D, BF, seed=5)
    spans = skv.Spans(i32([P] * B), i32([T] * B), i32([N] * B), T, rows)
    q = inputs.normal((B, rows, Hq, D), 6, dtype=BF).to(DEV)
    out, lse = torch.empty_like(q), torch.empty(B, Hq, rows, device=DEV)
    for mode in (skv.MASK_WINDOW_END, skv.MASK_WINDOW_START):
        skv.speechkv_prefill_attn(q, cache, spans, w, 1, 0, out, mask_mode=mode, lse=lse)
        visible = skv.visible_slots([[(P, T), (N, 0)]] * B, w, 1, 0, mode)
        got = torch.empty(B, Hkv, L, device=DEV)
        skv.speechkv_attn_weights(q, lse, cache, i32([L] * B), L, got, visible=visible)
        assert float((got.sum(2) - rows * Hq // Hkv).abs().max()) < 1e-3
        # row by row: nothing behind what it sees
        for i in (0, 5, 12, rows - 1):
            one = torch.empty(B, Hkv, L, device=DEV)
            skv.speechkv_attn_weights(q[:, i:i + 1], lse[:, :, i:i + 1], cache, i32([L] * B), L, one,
                                      visible=visible[:, i:i + 1].contiguous())
            n = int(visible[0, i])
            assert bool((one[:, :, n:] == 0).all()) and float((one[:, :, :n].sum(2) - Hq // Hkv).abs().max()) < 1e-5


def test_weights_of_rows_that_are_not_used_do_not_matter():
    """Queries, keys and lse of what no row sees may hold anything."""
    cache = make_cache(1, 100, 2, 64, BF, seed=8)
    q = inputs.normal((1, 40, 4, 64), 9, dtype=BF).to(DEV)
    lse = torch.full((1, 4, 40), 5.0, device=DEV)
    seen = [0 if i % 3 else 50 for i in range(40)]
    run = lambda: skv.speechkv_attn_weights(q, lse, cache, i32([100]), 100, out, visible=i32([seen]))  # noqa: E731
    out = torch.empty(1, 2, 100, device=DEV)
    run()
    want = out.clone()
    assert bool((want[0, :, 50:] == 0).all()) and bool((want[0, :, :50] > 0).all())
    for i, s in enumerate(seen):
        if not s:
            q[0, i] = float("nan")
            lse[0, :, i] = float("nan") if i % 2 else float("-inf")
    for c in range(50, 100):
        cache.k_pages[int(cache.block_table[0, c // 16]), :, c % 16] = float("inf")
    run()
    assert torch.equal(out, want)


def test_weights_without_a_page_stay():
    cache = make_cache(2, 64, 2, 128, BF, seed=3)
    cache.block_table[0, 1] = -1
    cache.block_table[1, 2] = 10 ** 5
    q, lse = inputs.normal((2, 1, 2, 128), 1, dtype=BF).to(DEV), torch.zeros(2, 2, 1, device=DEV)
    had = torch.rand(2, 2, 64, device=DEV)
    out = torch.zeros_like(had)
    skv.speechkv_attn_weights(q, lse, cache, i32([64, 40]), 64, out, weights=had)
    assert torch.equal(out[0, :, 16:32], had[0, :, 16:32]) and torch.equal(out[1, :, 32:40], had[1, :, 32:40])
    assert bool((out[0, :, :16] > had[0, :, :16]).all()) and bool((out[1, :, 40:] == 0).all())


# ------------------------------------------------------------------ eviction

EVICT = [
    # dtype, D, Hkv, page, lengths, keep, first, recent, layers
    (BF, 128, 8, 16, [400], [256], 4, 32, 1),
    (BF, 128, 2, 16, [0, 1, 2, 300, 64, 65], [5, 1, 1, 299, 64, 0], 0, 0, 3),
    (BF, 64, 4, 8, [1000, 513], [100, 512], 3, 7, 2),
    (F32, 128, 1, 64, [777], [400], 0, 500, 2),
    (F32, 64, 2, 256, [130, 128], [64, 127], 100, 3, 1),
    (BF, 128, 2, 16, [90] * 3, [40, 41, 90], 2, 5, 70),
    (BF, 64, 1, 16, [5000], [2500], 10, 100, 1),
    (BF, 128, 1, 32, [40, 9], [1, 8], 0, 1, 1),
    # choice and moves in one kernel; weights that stay in registers, and that do not
    (BF, 64, 8, 16, [2500] + [300 + 7 * i for i in range(15)], [200 + 20 * i for i in range(16)], 4, 16, 5),
    (F32, 128, 16, 8, [70, 20], [40, 30], 2, 3, 33),
]


class Evict:
    def __init__(self, case, seed=0, special=True):
        dt, D, Hkv, page, self.lens, self.keep, self.first, self.recent, n = EVICT[case]
        self.B, self.n, most = len(self.lens), n, max(self.lens + [1])
        # one pool for all layers
        pool = make_cache(self.B * n, most, Hkv, D, dt, page, seed=900 + case + seed)
        tables = pool.block_table.view(n, self.B, -1)
        self.caches = [skv.PagedKV(pool.k_pages, pool.v_pages, t) for t in tables]
        g = torch.Generator().manual_seed(case + seed)
        w = torch.exp(2 * torch.randn((n, self.B, Hkv, most + 3), generator=g))
        if special:
            kind = torch.randint(0, 12, w.shape, generator=g)
            for i, v in enumerate((0.0, -0.0, 1.0, float("nan"), float("inf"), float("-inf"), -2.5)):
                w[kind == i] = v
        self.weights = w.to(DEV)
        self.capacity, self.max_keep = most + 3, max(max(self.keep), 1)
        self.lens_t, self.pool = i32(self.lens), pool

    def want(self):
        """kept, weights_out, pools, lengths of every layer."""
        pools = [self.pool.k_pages.clone(), self.pool.v_pages.clone()]
        kept = torch.full((self.n, self.B, self.weights.shape[2], self.max_keep), -9, dtype=torch.int32)
        w_out = torch.full_like(self.weights, -3.0)
        ps = pools[0].shape[2]
        for i in range(self.n):
            t = self.caches[i].block_table
            for b, L in enumerate(self.lens):
                for g in range(self.weights.shape[2]):
                    w = self.weights[i, b, g, :L].cpu().numpy()
                    s = ref.kept_slots(w, self.keep[b], self.first, self.recent)
                    kept[i, b, g, :len(s)] = torch.tensor(s, dtype=torch.int32)
                    w_out[i, b, g, :L] = 0.0
                    st = torch.tensor(s, dtype=torch.long, device=DEV)
                    w_out[i, b, g, :len(s)] = self.weights[i, b, g, st]
                    j = torch.arange(len(s), device=DEV)
                    for x in pools:
                        x[t[b, j // ps].long(), g, j % ps] = x[t[b, st // ps].long(), g, st % ps].clone()
        return kept, w_out, pools, [min(a, b) for a, b in zip(self.lens, self.keep)]

    def run(self, w_out=None, kept=None, stream=None):
        lens_out = [i32([-1] * self.B) for _ in range(self.n)]
        if kept is None:
            kept, self.guard = guarded((self.n, self.B, self.weights.shape[2], self.max_keep), torch.int32, DEV, fill=-9)
        w_out = torch.full_like(self.weights, -3.0) if w_out is None else w_out
        stack = skv.EvictStack(self.caches, [self.lens_t] * self.n, lens_out, list(self.weights), list(w_out), list(kept))
        skv.speechkv_evict(stack, i32(self.keep), self.first, self.recent, stream=stream)
        torch.cuda.synchronize()
        return kept, w_out, lens_out


def bits(x):
    return x.contiguous().view(torch.int16 if x.element_size() == 2 else torch.int32)


@pytest.mark.parametrize("case", range(len(EVICT)))
@pytest.mark.parametrize("in_place", [False, True])
def test_evict(case, in_place):
    x = Evict(case)
    kept, w_out, pools, lens = x.want()
    if in_place:
        for b, L in enumerate(x.lens):
            w_out[:, b, :, L:] = x.weights[:, b, :, L:]
    got_kept, got_w, got_lens = x.run(w_out=x.weights if in_place else None)
    x.guard("kept")
    assert torch.equal(got_kept.cpu(), kept)
    assert all(t.tolist() == lens for t in got_lens)
    assert torch.equal(bits(got_w), bits(w_out))
    assert torch.equal(bits(x.pool.k_pages), bits(pools[0])) and torch.equal(bits(x.pool.v_pages), bits(pools[1]))


@pytest.mark.parametrize("value", [0.0, 1.0, float("nan"), float("inf")])
def test_evict_ties_go_to_the_lowest_slots(value):
    x = Evict(0)
    x.weights[:] = value
    kept, _, _ = x.run()
    n, f, r, L = 256, 4, 32, 400
    assert bool((kept[..., :n - r] == torch.arange(n - r, device=DEV)).all())
    assert bool((kept[..., n - r:] == torch.arange(L - r, L, device=DEV)).all())


def test_evict_lengths_and_pages_out_of_range():
    """Lengths beyond the table or the capacity are cut, keep_len beyond max_keep
    too; entries without a page, or whose place has none, are not moved."""
    x = Evict(5, special=False)
    x.n, x.caches, x.weights = 1, x.caches[:1], x.weights[:1].contiguous()
    t = x.caches[0].block_table.clone()
    for b in range(3):
        x.caches[0].block_table[b, 1] = -1
        x.caches[0].block_table[b, 4] = 10 ** 6
    k0, ps = x.pool.k_pages.clone(), 16
    x.lens_t, keep = i32([90, 2 ** 31 - 1, -3]), x.keep
    x.keep, x.max_keep = [40, 2 ** 31 - 1, 90], 41
    kept, w_out, lens_out = x.run()
    assert lens_out[0].tolist() == [40, 41, 0]
    cap = min(x.capacity, x.caches[0].block_table.shape[1] * ps)
    want = k0.clone()
    for b, L in ((0, 90), (1, cap)):
        for g in range(2):
            s = ref.kept_slots(x.weights[0, b, g, :L].cpu().numpy(), min(x.keep[b], 41), 2, 5)
            assert kept[0, b, g, :len(s)].tolist() == s
            for j, c in enumerate(s):
                if 1 not in (j // ps, c // ps) and 4 not in (j // ps, c // ps):
                    want[t[b, j // ps], g, j % ps] = k0[t[b, c // ps], g, c % ps]
    assert torch.equal(x.pool.k_pages, want) and keep


def test_evict_captured_and_on_another_stream():
    x = Evict(2)
    k0, v0 = x.pool.k_pages.clone(), x.pool.v_pages.clone()
    new = [x.weights.clone(), x.weights.flip(-1).contiguous(), torch.rand_like(x.weights)]
    kept, w_out, lens_out = x.run()
    stack = skv.EvictStack(x.caches, [x.lens_t] * x.n, lens_out, list(x.weights), list(w_out), list(kept))
    keep = i32(x.keep)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        skv.speechkv_evict(stack, keep, x.first, x.recent)
    side = torch.cuda.Stream()
    for w in new:
        x.weights.copy_(w)
        results = []
        for replay in (False, True):
            x.pool.k_pages.copy_(k0)
            x.pool.v_pages.copy_(v0)
            kept.fill_(-9)
            w_out.fill_(-3.0)
            torch.cuda.synchronize()
            if replay:
                graph.replay()
            else:
                skv.speechkv_evict(stack, keep, x.first, x.recent, stream=side)
            torch.cuda.synchronize()
            results.append([t.clone() for t in (kept, bits(w_out), x.pool.k_pages, x.pool.v_pages)])
        assert all(torch.equal(a, b) for a, b in zip(*results))


# ------------------------------------------------------------------ far away

def test_offsets_past_32_bits():
    """Pages and rows that lie more than 2^32 bytes into their tensors give what the
    same values near the start give."""
    Hq, Hkv, D, ps, pages = 4, 2, 128, 256, 34000  # 4.5 GB a pool
    k, v = (torch.empty((pages, Hkv, ps, D), dtype=BF, device=DEV) for _ in range(2))
    far, near = [pages - 1, 2, pages - 40, pages - 3], [0, 1, 2, 3]
    nk, nv = (inputs.normal((4, Hkv, ps, D), 30 + i, dtype=BF).to(DEV) for i in range(2))
    for i, p in enumerate(far):
        k[p], v[p] = nk[i], nv[i]
    L = 4 * ps - 9
    results = []
    for kk, vv, t in ((k, v, far), (nk, nv, near)):
        c = skv.PagedKV(kk, vv, i32([t]))
        mine = skv.PagedKV(kk, vv, i32([t[1:2], t[2:3], t[3:]]))
        q = inputs.normal((3, Hq, D), 40, dtype=BF).to(DEV)
        out, lse = torch.empty_like(q), torch.empty(3, Hq, device=DEV)
        need = skv.speechkv_shared_workspace_bytes(3, 1, 3, Hq, Hkv, D, L, 200)
        skv.speechkv_shared_attn(q, c, i32([L]), L, i32([0, 3]), 3, mine, i32([200, 3, 77]), 200, out, lse=lse,
                                 workspace=torch.empty(need, dtype=torch.uint8, device=DEV))
        gathered = []
        for rows in (q[:, None], q[:, None].expand(3, 20, Hq, D)):  # few rows, many rows
            n = rows.shape[1]
            w = torch.empty(1, Hkv, L, device=DEV)
            skv.speechkv_attn_weights(rows.reshape(1, 3 * n, Hq, D), lse[:, None].expand(3, n, Hq).reshape(3 * n, Hq).t()[None],
                                      c, i32([L]), L, w, visible=i32([[L - i for i in range(3 * n)]]))
            gathered.append(w)
        kept, n_out = torch.zeros((1, Hkv, 500), dtype=torch.int32, device=DEV), i32([0])
        skv.speechkv_evict(skv.EvictStack([c], [i32([L])], [n_out], [gathered[1]], [torch.empty_like(w)], [kept]), i32([500]),
                           4, 8)
        new = inputs.normal((1, 7, Hq + 2 * Hkv, D), 50, dtype=BF).to(DEV)
        skv.speechkv_norm_append_kv(None, new[:, :, Hq:Hq + Hkv], new[:, :, Hq + Hkv:], c, n_out)
        table = c.block_table[0, :2].long()
        results.append([out, lse, *gathered, kept, kk[table].clone(), vv[table].clone()])
    assert all(torch.equal(a, b) for a, b in zip(*results))
    # rows of a tensor that ends 4.5 GB behind its start, read and written in place
    flat = k.view(-1)
    rows = torch.as_strided(flat, (2, 3, 2, D), (flat.numel() - 3 * 2 * D, 2 * D, D, 1))
    x = inputs.normal((2, 3, 2, D), 60, dtype=BF).to(DEV)
    rows.copy_(x)
    want, dx, dwant = torch.empty_like(x), torch.empty_like(x), torch.empty_like(x)
    skv.speechkv_norm_rope(x, None, want, None)
    skv.speechkv_norm_rope_bwd(x, None, want, None, dwant, None)
    skv.speechkv_norm_rope_bwd(rows, None, want, None, dx, None)
    skv.speechkv_norm_rope(rows, None, rows, None)
    assert torch.equal(rows, want) and torch.equal(dx, dwant)


def test_weights_of_heads_that_lie_far_apart():
    # heads 1.4 GB apart: the rows of one load span more than 31 bits
    Hq, Hkv, D, S, L = 4, 1, 128, 40, 300
    apart = 7 * 10 ** 8
    cache = make_cache(1, L, Hkv, D, BF, 16, seed=90)
    q = inputs.normal((1, S, Hq, D), 91, dtype=BF).to(DEV)
    far = torch.as_strided(torch.empty(3 * apart + S * D, dtype=BF, device=DEV), (1, S, Hq, D), (0, D, apart, 1))
    far.copy_(q)
    lse = torch.full((1, Hq, S), 3.0, device=DEV)
    one, two = (torch.full((1, Hkv, L), -1.0, device=DEV) for _ in range(2))
    skv.speechkv_attn_weights(q, lse, cache, i32([L]), L, one)
    skv.speechkv_attn_weights(far, lse, cache, i32([L]), L, two)
    assert torch.equal(one, two) and bool((one >= 0).all())


# ------------------------------------------------------------- all together

def test_questions_about_a_recording_within_a_budget():
    """A run of the operators as a server uses them: a prompt is normed, rotated,
    pooled into the recording's cache and attended; its entries gather weight;
    two questions decode over the recording and their own entries and add what
    they look at; the recording is shortened and decoding goes on.  Every step
    against the plain form of the shortened cache."""
    P, T, N, w, Hq, Hkv, D, Q, steps = 6, 61, 9, 4, 4, 2, 128, 5, 3
    rows, L = P + T + N, P + 16 + N
    inv = (1e4 ** (-torch.arange(0, D, 2, dtype=torch.float64) / D)).float().to(DEV)
    gq, gk = (1 + 0.1 * torch.randn(D, device=DEV) for _ in range(2))
    qkv = inputs.normal((1, rows, Hq + 2 * Hkv, D), 1, dtype=BF).to(DEV)
    q, k, v = qkv[:, :, :Hq], qkv[:, :, Hq:Hq + Hkv], qkv[:, :, Hq + Hkv:]
    qn, kn = torch.empty((1, rows, Hq, D), dtype=BF, device=DEV), torch.empty((1, rows, Hkv, D), dtype=BF, device=DEV)
    pos = torch.arange(rows, dtype=torch.int32, device=DEV)[None]
    skv.speechkv_norm_rope(q, k, qn, kn, gq, gk, rope=skv.Rope(pos, inv))
    rec = make_cache(1, L, Hkv, D, BF, seed=2)
    spans = skv.Spans(i32([P]), i32([T]), i32([N]), T, rows)
    rec_len = i32([0])
    skv.speechkv_pool_kv(kn, v.contiguous(), spans, w, None, 1, 0, rec, rec_len)
    out, lse = torch.empty_like(qn), torch.empty(1, Hq, rows, device=DEV)
    skv.speechkv_prefill_attn(qn, rec, spans, w, 1, 0, out, lse=lse)
    weights = torch.zeros(1, Hkv, L, device=DEV)
    skv.speechkv_attn_weights(qn, lse, rec, rec_len, L, weights, visible=skv.visible_slots([[(P, T), (N, 0)]], w, 1, 0))
    assert rec_len.tolist() == [L] and abs(float(weights.sum()) - rows * Hq) < 1e-2

    own = make_cache(Q, steps, Hkv, D, BF, seed=3)
    own_len, start, total = i32([0] * Q), i32([0, Q]), L
    ws = torch.empty(skv.speechkv_shared_workspace_bytes(Q, 1, Q, Hq, Hkv, D, L, steps), dtype=torch.uint8, device=DEV)
    for step in range(steps):
        new = inputs.normal((Q, 1, Hq + 2 * Hkv, D), 10 + step, dtype=BF).to(DEV)
        qs = torch.empty((Q, 1, Hq, D), dtype=BF, device=DEV)
        skv.speechkv_norm_append_kv(new[:, :, :Hq], new[:, :, Hq:Hq + Hkv], new[:, :, Hq + Hkv:], own, own_len, qs, gq,
                                    gk, rope=skv.Rope(i32([[rows + step]] * Q), inv), cache_len_out=(nxt := i32([0] * Q)))
        own_len = nxt
        o, ls = torch.empty((Q, Hq, D), dtype=BF, device=DEV), torch.empty((Q, Hq), device=DEV)
        skv.speechkv_shared_attn(qs[:, 0], rec, rec_len, L, start, Q, own, own_len, steps, o, lse=ls, workspace=ws)
        pk, pv, ok, ov = (f64(x) for x in (rec.k_pages, rec.v_pages, own.k_pages, own.v_pages))
        for b in range(Q):
            sources = [ref.entries(pk, pv, f64(rec.block_table).astype(int), 0, total)[1:],
                       ref.entries(ok, ov, f64(own.block_table).astype(int), b, step + 1)[1:]]
            want, bound, l, lbound = ref.attention(f64(qs[b, 0]), sources, D ** -0.5, HALF[BF], 1088)
            check(o[b], want, bound, (step, b))
            check(ls[b], l, lbound, (step, b))
        # what all questions look at in the recording: one batch of Q rows
        before = f64(weights[0])
        skv.speechkv_attn_weights(qs.transpose(0, 1), ls.t()[None], rec, rec_len, L, weights, weights=weights,
                                  visible=i32([[L] * Q]))
        keys = ref.entries(pk, pk, f64(rec.block_table).astype(int), 0, total)[1]
        for g in range(Hkv):
            heads = slice(g * Hq // Hkv, (g + 1) * Hq // Hkv)
            want, bound = ref.gathered(f64(qs[:, 0, heads]).reshape(-1, D), f64(ls[:, heads]).reshape(-1),
                                       np.full(Q * Hq // Hkv, total), keys[:, g], D ** -0.5, before[g, :total])
            check(weights[0, g, :total], want, bound, (step, g))
        if step == 1:  # the recording gets shorter
            slots = [ref.kept_slots(weights[0, g].cpu().numpy(), 20, 4, 3) for g in range(Hkv)]
            kept, short = torch.zeros((1, Hkv, 20), dtype=torch.int32, device=DEV), i32([0])
            rows_before = ref.entries(f64(rec.k_pages), f64(rec.v_pages), f64(rec.block_table).astype(int), 0, L)[1:]
            skv.speechkv_evict(skv.EvictStack([rec], [rec_len], [short], [weights], [weights], [kept]), i32([20]), 4, 3)
            assert short.tolist() == [20] and kept[0].tolist() == slots
            rec_len, total = short, 20
            rows_after = ref.entries(f64(rec.k_pages), f64(rec.v_pages), f64(rec.block_table).astype(int), 0, 20)[1:]
            for g in range(Hkv):
                for x, y in zip(rows_before, rows_after):
                    assert np.array_equal(x[slots[g], g], y[:, g])
            assert bool((weights[0, :, 20:] == 0).all())
