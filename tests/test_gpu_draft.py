"""The steps of several new tokens on the GPU against plain 64-bit forms
(tests/draft_ref.py, which derives the bounds)."""
import numpy as np
import pytest
import torch

import draft_ref as ref
from draft_ref import HALF, U, f64
from gpu_case import guarded, launches
from paper_2607_06827_amd import inputs
from paper_2607_06827_amd import speechkv as skv

pytestmark = [pytest.mark.gpu,
              pytest.mark.skipif(not torch.cuda.is_available(), reason="needs a GPU")]

DEV = "cuda"
BF, F32 = torch.bfloat16, torch.float32


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def make_cache(B, slots, Hkv, D, dtype, page=16, seed=0, spare=3):
    """A cache of random pages with room for `slots` entries per sequence."""
    table, total = inputs.block_table(B, max(1, -(-slots // page)), seed, shuffle=True, spare_pages=spare)
    k = inputs.normal((total, Hkv, page, D), seed + 1, dtype=dtype).to(DEV)
    v = inputs.normal((total, Hkv, page, D), seed + 2, dtype=dtype).to(DEV)
    return skv.PagedKV(k, v, table.to(DEV))


def rows_of(cache, b, first, n):
    """K and V [n, Hkv, D] of cache slots first .. first + n."""
    ps = cache.k_pages.shape[2]
    s = torch.arange(first, first + n, device=DEV)
    page = cache.block_table[b, s // ps].long()
    return cache.k_pages[page, :, s % ps], cache.v_pages[page, :, s % ps]


# ------------------------------------------------------------------- append

APPEND = [
    # dtype, D, Hq, Hkv, B, S, page, rot, pairs, lens, new, strides, far
    (BF, 128, 16, 8, 1, 1, 16, 128, False, [166], None, "fused", 0),
    (BF, 128, 16, 8, 3, 7, 16, 128, False, [0, 31, 250], [7, 3, 0], "fused", 0),
    (BF, 64, 4, 4, 2, 33, 8, 32, True, [5, 1], None, "dense", 10 ** 6),
    (F32, 64, 8, 1, 2, 5, 64, 16, True, [63, 64], [5, 1], "fused", 0),
    (F32, 128, 8, 2, 4, 65, 128, 128, False, [1, 0, 17, 100], [65, 64, 2, 1], "wide", 40000),
    (F32, 128, 4, 2, 1, 300, 256, 96, False, [3], None, "dense", 2 ** 31 - 400),
    (BF, 64, 0, 2, 2, 9, 16, 0, False, [7, 8], [4, 9], "wide", 0),
    (BF, 128, 2, 2, 65, 2, 32, 48, True, [i % 9 for i in range(65)], [i % 3 for i in range(65)], "fused", 100),
]


@pytest.mark.parametrize("case", range(len(APPEND)))
def test_append(case):
    dt, D, Hq, Hkv, B, S, page, rot, pairs, lens, new, strides, far = APPEND[case]
    cache = make_cache(B, max(lens) + S, Hkv, D, dt, page, seed=100 + case)
    n_new = new or [S] * B
    H = Hq + 2 * Hkv
    if strides == "fused":
        x = inputs.normal((B, S, H, D), 1, dtype=dt).to(DEV)
        q, k, v = x[:, :, :Hq], x[:, :, Hq:Hq + Hkv], x[:, :, Hq + Hkv:]
    elif strides == "wide":  # heads outermost, rows apart
        x = inputs.normal((H, B, S + 2, D + 16), 1, dtype=dt).to(DEV).permute(1, 2, 0, 3)[:, 1:S + 1, :, :D]
        q, k, v = x[:, :, :Hq], x[:, :, Hq:Hq + Hkv], x[:, :, Hq + Hkv:]
    else:
        q, k, v = (inputs.normal((B, S, h, D), 1 + h, dtype=dt).to(DEV) for h in (Hq, Hkv, Hkv))
    pos = (torch.arange(S)[None] + far + torch.arange(B)[:, None] * 3).to(torch.int32)
    inv = (1e4 ** (-torch.arange(0, rot, 2, dtype=torch.float64) / max(rot, 1))).float()
    k0, v0 = cache.k_pages.clone(), cache.v_pages.clone()
    q_out, guard = guarded((B, S, max(Hq, 1), D), dt, DEV, fill=-7.0)
    out_len = i32([-1] * B)
    skv.speechkv_append_kv(k, v, cache, i32(lens), positions=pos.to(DEV) if rot else None,
                           inv_freq=inv.to(DEV) if rot else None, rope=skv.ROPE_PAIRS if pairs else skv.ROPE_HALVES,
                           q=q if Hq else None, q_out=q_out if Hq else None, new_len=None if new is None else i32(new),
                           cache_len_out=out_len)
    guard("append q_out")
    assert out_len.tolist() == [a + b for a, b in zip(lens, n_new)]

    def check(got, src, p):
        want, size, err = ref.rotate(f64(src), p, inv.double().numpy(), pairs)
        bound = np.where(np.arange(D) < rot, (7 * U + err) * size, 0.0)
        bound = (bound + HALF[dt] * (np.abs(want) + bound) * (np.arange(D) < rot)) * (1 + 1e-6)
        assert np.all(np.abs(f64(got) - want) <= bound), np.max(np.abs(f64(got) - want) - bound)

    touched = torch.zeros(cache.k_pages.shape[0], cache.k_pages.shape[2], dtype=torch.bool, device=DEV)
    for b in range(B):
        n, p = n_new[b], pos[b, :n_new[b]].numpy()
        gk, gv = rows_of(cache, b, lens[b], n)
        check(gk, k[b, :n], p)
        assert torch.equal(gv, v[b, :n])
        if Hq:
            check(q_out[b, :n], q[b, :n], p)
            assert bool((q_out[b, n:] == -7.0).all())
        s = torch.arange(lens[b], lens[b] + n, device=DEV)
        touched[cache.block_table[b, s // page].long(), s % page] = True
    # every other row of the pools is as it was
    same = ~touched[:, None, :, None]
    assert torch.equal(torch.where(same, cache.k_pages, k0), k0) and torch.equal(torch.where(same, cache.v_pages, v0), v0)


def test_append_rotates_queries_in_place():
    cache = make_cache(2, 40, 2, 128, BF)
    q, k, v = (inputs.normal((2, 5, h, 128), 9 + h, dtype=BF).to(DEV) for h in (4, 2, 2))
    pos, inv = torch.arange(10, dtype=torch.int32, device=DEV).view(2, 5) + 1000, torch.rand(64).to(DEV)
    out = torch.empty_like(q)
    skv.speechkv_append_kv(k, v, cache, i32([3, 30]), pos, inv, q=q, q_out=out)
    skv.speechkv_append_kv(k, v, cache, i32([3, 30]), pos, inv, q=q, q_out=q)
    assert torch.equal(q, out)


def test_append_skips_what_has_no_page():
    """Bad table entries, slots past the table and negative lengths: neither
    read nor written out of range; the other tokens are stored."""
    B, S, Hkv, D, page = 4, 6, 2, 64, 8
    cache = make_cache(B, 16, Hkv, D, BF, page)
    cache.block_table[0, 0] = -1
    cache.block_table[1, 1] = cache.k_pages.shape[0]
    lens = [5, 5, 13, -4]
    k, v = (inputs.normal((B, S, Hkv, D), 20 + i, dtype=BF).to(DEV) for i in range(2))
    k0, t = cache.k_pages.clone(), cache.block_table.tolist()
    out_len = i32([0] * B)
    skv.speechkv_append_kv(k, v, cache, i32(lens), new_len=i32([6, 6, 99, 2]), cache_len_out=out_len)
    assert out_len.tolist() == [11, 11, 19, 2]
    want = k0.clone()
    for b in range(B):
        for i in range([6, 6, 6, 2][b]):
            slot = max(lens[b], 0) + i
            if slot < 16 and 0 <= t[b][slot // page] < k0.shape[0]:
                want[t[b][slot // page], :, slot % page] = k[b, i]
    assert torch.equal(cache.k_pages, want)


# --------------------------------------------------------------------- tree

def random_tree(rng, n):
    return [-1] + [int(rng.integers(max(0, i // 3 - 1), i)) for i in range(1, n)]


TREE = [
    # dtype, D, Hkv, G, page, lens, n, nodes, mask, splits
    (BF, 128, 2, 2, 16, [166], 8, None, "tree", 0),
    (BF, 128, 1, 1, 16, [0], 1, None, "chain", 0),
    (BF, 128, 1, 1, 16, [1], 1, None, "tree", 1),
    (BF, 128, 1, 2, 16, [31, 32, 33], 16, None, "tree", 1),
    (BF, 128, 2, 4, 8, [0, 7, 8, 64, 129], 9, [9, 0, 1, 5, 9], "tree", 1),
    (BF, 64, 2, 2, 64, [100, 3, 0], 33, [33, 32, 31], "shared", 0),
    (BF, 64, 1, 8, 16, [77, 200], 40, [40, 17], "tree", 3),
    (BF, 64, 4, 1, 256, [255, 257], 5, None, "chain", 2),
    (BF, 128, 1, 8, 32, [45, 300], 70, [61, 70], "chain", 0),
    (BF, 128, 1, 2, 16, [1500], 65, None, "tree", 7),
    (BF, 128, 1, 2, 128, [700, 20], 64, None, "dag", 5),
    (BF, 128, 3, 2, 16, [40, 111, 3, 64], 7, [7, 2, 7, 1], "tree", 1),
    (BF, 64, 5, 4, 16, [0, 2, 600], 50, [50, 1, 0], "tree", 3),
    (BF, 128, 1, 1, 16, [90], 1024, None, "chain", 0),
    (BF, 64, 1, 1, 8, [3], 1024, [1000], "tree", 2),
    (F32, 64, 2, 2, 16, [166, 0, 5], 8, [8, 8, 2], "tree", 0),
    (F32, 128, 1, 4, 8, [33, 1, 90], 33, [1, 33, 20], "dag", 1),
    (F32, 128, 2, 1, 32, [500], 21, None, "chain", 4),
    (F32, 64, 1, 8, 16, [64], 40, None, "tree", 2),
]


def tree_case(case, seed):
    dt, D, Hkv, G, page, lens, n, nodes, mask, splits = case
    rng = np.random.default_rng(seed)
    B = len(lens)
    cache = make_cache(B, max(lens) + n, Hkv, D, dt, page, seed)
    q = inputs.normal((B, n, Hkv * G, D), seed + 5, dtype=dt).to(DEV)
    if mask == "chain":
        words, see = None, lambda b, i, j: j <= i
    elif mask == "dag":  # any nodes, not always itself, an empty row
        bits = rng.random((B, n, n)) < 0.4
        bits[:, n // 2] = False
        words = np.zeros((B, n, -(-n // 32)), dtype=np.uint32)
        for b, i, j in np.argwhere(bits):
            words[b, i, j // 32] |= np.uint32(1 << (j % 32))
        words, see = torch.from_numpy(words.view(np.int32)).to(DEV), lambda b, i, j: bits[b, i, j]
    else:
        trees = [random_tree(rng, n) for _ in range(1 if mask == "shared" else B)]
        up = [ref.ancestors(t) for t in trees]
        words = skv.tree_mask(trees[0] if mask == "shared" else trees)
        see = (lambda b, i, j: j in up[0][i]) if mask == "shared" else lambda b, i, j: j in up[b][i]
    return cache, q, words, see, lens, nodes or [n] * B


def run_tree(cache, q, words, lens, nodes, n, splits=0, out=None, ws=None, slack=0):
    B, _, Hq, D = q.shape
    Hkv = cache.k_pages.shape[1]
    out = torch.full_like(q, float("nan")) if out is None else out
    bound = min(max(lens) + slack, cache.block_table.shape[1] * cache.k_pages.shape[2])
    need = skv.speechkv_tree_workspace_bytes(B, n, Hq, Hkv, D, bound, splits)
    guard = lambda what: None  # noqa: E731
    if ws is None:
        ws, guard = guarded((max(need, 16) // 4,), F32, DEV)
    skv.speechkv_tree_attn(q, cache, i32(lens), bound, out, tree_mask=words,
                           num_nodes=None if nodes == [n] * B else i32(nodes), num_splits=splits, workspace=ws)
    guard("tree workspace")
    return out


def check_tree(out, cache, q, see, lens, nodes, what=""):
    k, v = f64(cache.k_pages), f64(cache.v_pages)
    D = q.shape[3]
    want, bound = ref.tree(f64(q), k, v, cache.block_table.cpu().numpy(), [max(0, x) for x in lens], nodes, see,
                           float(np.float32(D ** -0.5)), HALF[q.dtype])
    got = f64(out)
    assert np.array_equal(np.isnan(got), np.isnan(want)), what
    live = ~np.isnan(want)
    worst = np.max(np.abs(got[live] - want[live]) / (bound[live] + 1e-300), initial=0.0)
    print(f"{what} error / bound {worst:.3f}", flush=True)
    assert worst <= 1.0, what


@pytest.mark.parametrize("case", range(len(TREE)))
def test_tree(case):
    n, splits = TREE[case][6], TREE[case][9]
    cache, q, words, see, lens, nodes = tree_case(TREE[case], 300 + 10 * case)
    out, guard = guarded(q.shape, q.dtype, DEV)
    run_tree(cache, q, words, lens, nodes, n, splits, out, slack=case % 3 * 40)
    guard("tree out")
    check_tree(out, cache, q, see, lens, nodes, f"case {case}")
    again = run_tree(cache, q, words, lens, nodes, n, splits, slack=case % 3 * 40)
    assert torch.equal(again.nan_to_num(), out.nan_to_num())  # (rows that are not written are NaN)


@pytest.mark.parametrize("dt", [BF, F32])
def test_tree_splits_agree(dt):
    """Every split count, also more ranges than keys, gives the same values."""
    case = (dt, 128, 2, 2, 16, [210, 0, 95], 11, [11, 3, 0], "tree", 0)
    cache, q, words, see, lens, nodes = tree_case(case, 77)
    for s in (1, 2, 3, 5, 16, 300):
        out = run_tree(cache, q, words, lens, nodes, 11, s)
        check_tree(out, cache, q, see, lens, nodes, f"{s} splits")


SHAPES = [
    # dtype, D, Hkv, G, B, longest, n, mask, splits, rows of a block
    (BF, 128, 8, 2, 33, 70, 32, "tree", 1, 64),
    (BF, 128, 8, 2, 33, 70, 32, "tree", 5, 64),
    (BF, 128, 8, 8, 16, 90, 70, "chain", 1, 128),
    (BF, 128, 8, 8, 16, 90, 70, "dag", 9, 128),
    (BF, 64, 8, 2, 70, 40, 40, "dag", 1, 128),
    (BF, 64, 8, 2, 70, 300, 32, "shared", 2, 64),
    (F32, 128, 4, 4, 30, 30, 64, "tree", 1, 128),
    (F32, 128, 4, 4, 24, 50, 40, "chain", 7, 128),
    (F32, 64, 8, 2, 70, 10, 32, "tree", 1, 64),
    (F32, 128, 8, 2, 33, 30, 32, "chain", 1, 64),
    (F32, 64, 8, 8, 20, 20, 50, "dag", 3, 128),
    (BF, 128, 16, 1, 3, 90, 1024, "tree", 1, 128),  # the longest mask rows, of one head each
    (F32, 128, 8, 2, 2, 30, 1024, "tree", 1, 128),
]


@pytest.mark.parametrize("case", range(len(SHAPES)))
def test_tree_block_shapes(case):
    """Calls whose blocks hold 64 and 128 rows, with tiles of several steps,
    splits behind the last key and values that are not finite."""
    dt, D, Hkv, G, B, longest, n, mask, splits, rows = SHAPES[case]
    rng = np.random.default_rng(case)
    lens = [longest] + [int(x) for x in rng.integers(0, longest + 1, B - 1)]
    nodes = [n] + [int(x) for x in rng.integers(0, n + 1, B - 1)]
    cache, q, words, see, lens, nodes = tree_case((dt, D, Hkv, G, 16, lens, n, nodes, mask, 0), 700 + case)
    out = run_tree(cache, q, words, lens, nodes, n, splits)
    units = B * Hkv * splits
    on_gpu, count, ws = i32(lens), i32(nodes), torch.empty(1 << 30, dtype=torch.uint8, device=DEV)
    first = launches(lambda: skv.speechkv_tree_attn(q, cache, on_gpu, longest, out, tree_mask=words, num_nodes=count,
                                                    num_splits=splits, workspace=ws))[0]
    assert first == ((units + 7) // 8 * 8 * -(-n * G // rows), 256)
    check_tree(out, cache, q, see, lens, nodes, f"case {case}")
    # a value that is not finite in the second node: infinite where it is seen
    at = [(b, *ref.slot_row(cache.block_table.cpu().numpy(), b, lens[b] + 1, 16, cache.v_pages.shape[0]))
          for b in range(B) if nodes[b] > 1]
    for b, page, row in at:
        cache.v_pages[page, :, row, 3] = float("-inf")
    far = run_tree(cache, q, words, lens, nodes, n, splits)
    hit = torch.zeros(out.shape[:2], dtype=torch.bool)
    for b, _, _ in at:
        hit[b, :nodes[b]] = torch.tensor([bool(see(b, i, 1)) for i in range(nodes[b])])
    assert hit.any() and torch.equal(torch.isinf(far[..., 3]).all(2).cpu(), hit)
    for b, page, row in at:
        cache.v_pages[page, :, row, 3] = 0.0
    zero = run_tree(cache, q, words, lens, nodes, n, splits)
    far[..., 3][hit.to(DEV)] = zero[..., 3][hit.to(DEV)]
    assert torch.equal(far.nan_to_num(7.0), zero.nan_to_num(7.0))


@pytest.mark.parametrize("dt,splits", [(BF, 1), (BF, 4), (F32, 1), (F32, 4)])
def test_tree_what_is_not_seen_does_not_matter(dt, splits):
    """Infinities and NaN in nodes that a row does not see, behind the last
    node, in pages that no table names: the row's output has none of them; a
    row that sees such a node has."""
    n, lens, nodes = 12, [37, 0, 64], [12, 7, 5]
    case = (dt, 128, 2, 2, 16, lens, n, nodes, "tree", 0)
    cache, q, words, see, lens, nodes = tree_case(case, 91)
    bad = {0: 4, 1: 3, 2: 2}  # one node of each sequence
    want, bound = ref.tree(f64(q), f64(cache.k_pages), f64(cache.v_pages), cache.block_table.cpu().numpy(), lens,
                           nodes, see, float(np.float32(128 ** -0.5)), HALF[dt])
    ps = 16
    named = set()
    for b in range(3):
        for slot in range(lens[b] + nodes[b]):
            named.add((int(cache.block_table[b, slot // ps]), slot % ps))
    for page in range(cache.k_pages.shape[0]):
        for r in range(ps):
            if (page, r) not in named:
                cache.k_pages[page, :, r], cache.v_pages[page, :, r] = float("nan"), float("inf")
    for b, j in bad.items():
        slot = lens[b] + j
        page, r = int(cache.block_table[b, slot // ps]), slot % ps
        cache.v_pages[page, 0, r, 5], cache.v_pages[page, 1, r] = float("inf"), float("nan")
        cache.k_pages[page, 1, r, 7] = float("nan")
    out = f64(run_tree(cache, q, words, lens, nodes, n, splits))
    G = 2
    for b, j in bad.items():
        for i in range(nodes[b]):
            near = np.abs(out[b, i] - want[b, i]) <= bound[b, i]
            if see(b, i, j):
                assert np.isinf(out[b, i, :G, 5]).all() and np.isnan(out[b, i, G:]).all(), (b, i)
                near[:G, 5] = near[G:] = True
            assert near.all(), (b, i)


@pytest.mark.parametrize("dt", [BF, F32])
def test_tree_skips_what_has_no_page(dt):
    """Bad table entries and lengths beyond the table or below 0 count as keys
    that no node sees."""
    case = (dt, 128, 1, 2, 8, [50, 60, 64, 20], 9, [9, 9, 5, 9], "tree", 0)
    cache, q, words, see, lens, nodes = tree_case(case, 55)
    cache.block_table[0, 2], cache.block_table[0, 7], cache.block_table[1, 0] = -1, 2 ** 31 - 1, -2 ** 31
    lens = [50, 60, 70, -3]  # (the table of sequence 2 ends at slot 73)
    cache.block_table = cache.block_table[:, :9].contiguous()
    for splits in (1, 3):
        out = run_tree(cache, q, words, lens, nodes, 9, splits)
        check_tree(out, cache, q, see, [50, 60, 70, 0], nodes, f"{splits} splits")


def test_tree_equals_decoding_one_by_one():
    """A chain of drafted tokens gives what decode steps give, one by one."""
    B, Hq, Hkv, D, n, L = 3, 8, 4, 128, 6, [40, 7, 129]
    cache = make_cache(B, max(L) + n, Hkv, D, F32, seed=8)
    q, k, v = (inputs.normal((B, n, h, D), 30 + h + i, dtype=F32).to(DEV) for i, h in enumerate((Hq, Hkv, Hkv)))
    skv.speechkv_append_kv(k, v, cache, i32(L))
    out = run_tree(cache, q, None, L, [n] * B, n)
    for i in range(n):
        step = torch.empty(B, Hq, D, device=DEV)
        skv.speechkv_decode_attn(q[:, i].contiguous(), cache, i32([x + i + 1 for x in L]), max(L) + i + 1, step,
                                 num_splits=1)
        assert torch.allclose(out[:, i], step, rtol=1e-5, atol=1e-5)


def test_tree_far_offsets():
    """Pages behind 2^32 bytes and 2^31 elements of a pool."""
    Hkv, D, page, total = 8, 128, 64, 36000  # 4.7 GB a pool, 2.36e9 elements
    k = torch.empty((total, Hkv, page, D), dtype=BF, device=DEV)
    v = torch.empty_like(k)
    table = i32([[35999, 3, 35000, 34000]])
    for p in table[0].tolist():
        k[p].normal_()
        v[p].normal_()
    cache = skv.PagedKV(k, v, table)
    n, L = 5, 200
    q, kn, vn = (inputs.normal((1, n, h, D), 40 + i, dtype=BF).to(DEV) for i, h in enumerate((16, 8, 8)))
    skv.speechkv_append_kv(kn, vn, cache, i32([L]))
    out = run_tree(cache, q, None, [L], [n], n)
    small = skv.PagedKV(k[table[0].long()].clone(), v[table[0].long()].clone(), i32([[0, 1, 2, 3]]))
    stack = skv.CacheStack([cache, small], [i32([L])] * 2, [i32([0]), i32([0])])
    check_tree(out, small, q, lambda b, i, j: j <= i, [L], [n])
    skv.speechkv_tree_commit(stack, i32([[0, 3, 4]]), i32([3]), n)
    assert torch.equal(k[table[0].long()], small.k_pages) and torch.equal(v[table[0].long()], small.v_pages)
    del k, v, cache
    torch.cuda.empty_cache()


# ------------------------------------------------------------------- commit

COMMIT = [
    # dtype, D, Hkv, page, lens per layer, n, path, path_len
    (BF, 128, 8, 16, [[166]], 8, [[0, 2, 5, 7]], [4]),
    (BF, 64, 2, 8, [[0, 7, 30], [3, 64, 9]], 9, [[1, 2, 3], [0, 0, 0], [8, 0, 8]], [3, 0, 2]),
    (F32, 128, 3, 64, [[60, 1]], 40, [[39] * 7, [5, 4, 3, 2, 1, 0, 6]], [7, 7]),
    (F32, 64, 1, 16, [[5], [9], [0]], 3, [[2, 1, 0]], [3]),
    (BF, 128, 2, 32, [[17]], 1024, [list(range(1023, -1, -1))], [1024]),
    (F32, 128, 1, 256, [[100, 3]], 600, [list(range(1, 600)), list(range(0, 599))], [599, 300]),
    (BF, 64, 2, 16, [[7]] * 35, 5, [[1, 4, -1, 9, 2 ** 31 - 1]], [5]),
]


@pytest.mark.parametrize("case", range(len(COMMIT)))
def test_commit(case):
    dt, D, Hkv, page, lens, n, path, plen = COMMIT[case]
    B = len(path)
    caches = [make_cache(B, max(L) + n, Hkv, D, dt, page, seed=50 * i + case) for i, L in enumerate(lens)]
    want = []
    for c, L in zip(caches, lens):
        k, v = c.k_pages.clone(), c.v_pages.clone()
        for b in range(B):
            gk, gv = (x.clone() for x in rows_of(c, b, L[b], n))
            for j in range(plen[b]):
                if 0 <= path[b][j] < n:
                    s = L[b] + j
                    pg, r = int(c.block_table[b, s // page]), s % page
                    k[pg, :, r], v[pg, :, r] = gk[path[b][j]], gv[path[b][j]]
        want.append((k, v))
    outs = [i32([-1] * B) if i % 2 == 0 else None for i in range(len(lens))]
    stack = skv.CacheStack(caches, [i32(L) for L in lens], outs)
    skv.speechkv_tree_commit(stack, i32(path), i32(plen), n)
    for c, L, out, (k, v) in zip(caches, lens, outs, want):
        assert torch.equal(c.k_pages, k) and torch.equal(c.v_pages, v)
        assert out is None or out.tolist() == [a + b for a, b in zip(L, plen)]


def test_commit_skips_what_has_no_page():
    cache = make_cache(3, 16, 2, 64, BF, 8)
    cache.block_table[0, 0] = -5
    cache.block_table[1, 1] = 10 ** 6
    k0, t, lens = cache.k_pages.clone(), cache.block_table.tolist(), [5, 5, 14]
    out = i32([0] * 3)
    skv.speechkv_tree_commit(skv.CacheStack([cache], [i32(lens)], [out]), i32([[1, 4, 5]] * 3), i32([3, 99, 3]), 6)
    assert out.tolist() == [8, 8, 17]
    want, ok = k0.clone(), lambda b, s: s < 16 and 0 <= t[b][s // 8] < k0.shape[0]
    for b in range(3):
        for j, p in enumerate([1, 4, 5]):
            if ok(b, lens[b] + p) and ok(b, lens[b] + j):
                want[t[b][(lens[b] + j) // 8], :, (lens[b] + j) % 8] = k0[t[b][(lens[b] + p) // 8], :, (lens[b] + p) % 8]
    assert torch.equal(cache.k_pages, want)


# ------------------------------------------------------------------ together

class Step:
    """One pass of a serving program over several layers: append, attend,
    commit, with fixed buffers, so that it can be captured."""

    def __init__(self, layers=2, B=3, n=10, Hq=8, Hkv=4, D=64, dt=BF, seed=0, room=64):
        rng = np.random.default_rng(seed)
        self.n, self.B, self.layers = n, B, layers
        self.lens = [i32(rng.integers(0, 40, B)) for _ in range(layers)]
        self.next = [torch.zeros_like(x) for x in self.lens]
        self.caches = [make_cache(B, 40 + room, Hkv, D, dt, 16, seed + 9 * i) for i in range(layers)]
        x = inputs.normal((layers, B, n, Hq + 2 * Hkv, D), seed + 3, dtype=dt).to(DEV)
        self.q, self.k, self.v = x[..., :Hq, :], x[..., Hq:Hq + Hkv, :], x[..., Hq + Hkv:, :]
        self.parents = [random_tree(rng, n) for _ in range(B)]
        self.mask = skv.tree_mask(self.parents)
        depth = [[len(s) - 1 for s in ref.ancestors(t)] for t in self.parents]
        self.pos = i32([[500 + 7 * b + d for d in depth[b]] for b in range(B)])
        self.inv = torch.rand(D // 2, generator=torch.Generator().manual_seed(seed)).to(DEV)
        leaf = [max(range(n), key=lambda i: depth[b][i]) for b in range(B)]
        paths = [sorted(ref.ancestors(t)[leaf[b]]) for b, t in enumerate(self.parents)]
        most = max(map(len, paths))
        self.path = i32([p + [0] * (most - len(p)) for p in paths])
        self.path_len = i32([len(p) for p in paths])
        self.q_rot = torch.zeros(layers, B, n, Hq, D, dtype=dt, device=DEV)
        self.out = torch.zeros_like(self.q_rot)
        need = skv.speechkv_tree_workspace_bytes(B, n, Hq, Hkv, D, 40, 3)
        self.ws = torch.empty(need, dtype=torch.uint8, device=DEV)
        self.stack = skv.CacheStack(self.caches, self.lens, self.next)

    def run(self, splits=3):
        for i, c in enumerate(self.caches):
            skv.speechkv_append_kv(self.k[i], self.v[i], c, self.lens[i], self.pos, self.inv, q=self.q[i],
                                   q_out=self.q_rot[i])
            skv.speechkv_tree_attn(self.q_rot[i], c, self.lens[i], 40, self.out[i], tree_mask=self.mask,
                                   num_splits=splits, workspace=self.ws)
        skv.speechkv_tree_commit(self.stack, self.path, self.path_len, self.n)

    def state(self):
        return [x.clone() for x in [self.out, *self.next, *(c.k_pages for c in self.caches),
                                    *(c.v_pages for c in self.caches)]]


def test_a_whole_step_equals_accepting_the_tokens_one_by_one():
    """append, tree_attn and commit leave the cache as appending only the
    accepted tokens would, and the accepted nodes' outputs are those of decode
    steps over that cache."""
    s = Step(dt=F32, seed=4)
    plain = [skv.PagedKV(c.k_pages.clone(), c.v_pages.clone(), c.block_table) for c in s.caches]
    s.run()
    for i, c in enumerate(plain):
        for b in range(s.B):
            m = int(s.path_len[b])
            for j in range(m):  # one token of one sequence at a time
                node = int(s.path[b, j])
                one = slice(node, node + 1)
                row = lambda x: x[i, b:b + 1, one]  # noqa: E731
                view = skv.PagedKV(c.k_pages, c.v_pages, c.block_table[b:b + 1].contiguous())
                L = int(s.lens[i][b]) + j
                qr = torch.empty(1, 1, *s.q.shape[3:], device=DEV)
                skv.speechkv_append_kv(row(s.k), row(s.v), view, i32([L]), s.pos[b:b + 1, one].contiguous(), s.inv,
                                       q=row(s.q), q_out=qr)
                out = torch.empty_like(qr[:, 0])
                skv.speechkv_decode_attn(qr[:, 0], view, i32([L + 1]), L + 1, out, num_splits=1)
                assert torch.allclose(s.out[i, b, node], out[0], rtol=1e-5, atol=1e-5)
            assert int(s.next[i][b]) == int(s.lens[i][b]) + m
            for x, y in zip(rows_of(c, b, 0, int(s.next[i][b])), rows_of(s.caches[i], b, 0, int(s.next[i][b]))):
                assert torch.equal(x, y)


def test_a_captured_step_replays_as_it_runs():
    """Two captured steps that share no buffer, replayed between eager work,
    give the eager bits every time."""
    want = []
    for seed in (1, 2):
        e = Step(seed=seed)
        e.run()
        want.append(e.state())
    steps, graphs, fresh = [], [], []
    for seed in (1, 2):
        st = Step(seed=seed)
        fresh.append([(c.k_pages.clone(), c.v_pages.clone()) for c in st.caches])
        side = torch.cuda.Stream()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=side):
            st.run()
        steps.append(st)
        graphs.append(g)
    for turn in range(4):
        for st, g, start, w in zip(steps, graphs, fresh, want):
            for c, (k, v) in zip(st.caches, start):
                c.k_pages.copy_(k)
                c.v_pages.copy_(v)
            st.out.zero_()
            g.replay()
            _ = torch.rand(1 << 16, device=DEV).sum()
            torch.cuda.synchronize()
            for x, y in zip(st.state(), w):
                assert torch.equal(x, y), turn


def test_steps_on_two_streams_do_not_meet():
    want = []
    for seed in (5, 6):
        e = Step(seed=seed)
        e.run()
        want.append(e.state())
    steps = [Step(seed=5), Step(seed=6)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for st, s in zip(steps, streams):
        with torch.cuda.stream(s):
            st.run()
    torch.cuda.synchronize()
    for st, w in zip(steps, want):
        for x, y in zip(st.state(), w):
            assert torch.equal(x, y)
