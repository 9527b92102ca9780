"""speechkv_tree_attn over caches long enough that a block works out its
addresses anew (every sixteen steps), in blocks of 32, 64 and 128 rows, with
pages of 8 to 128 rows and pages that are missing in the middle of a cache and
at its end, on the GPU against the 64-bit form."""
import numpy as np
import pytest
import torch

import draft_ref as ref
from gpu_case import guarded, launches
from paper_2607_06827_amd import speechkv as skv
from test_gpu_draft import BF, DEV, F32, check_tree, i32, run_tree, tree_case

pytestmark = [pytest.mark.gpu,
              pytest.mark.skipif(not torch.cuda.is_available(), reason="needs a GPU")]

CASES = [
    # dtype, D, Hkv, G, page, B, longest, n, mask, splits, rows of a block
    (BF, 128, 1, 2, 16, 2, 4500, 8, "tree", 1, 32),
    (BF, 64, 1, 2, 64, 2, 4500, 8, "dag", 1, 32),
    (BF, 128, 2, 1, 8, 2, 4600, 9, "chain", 2, 32),
    (F32, 128, 1, 2, 8, 2, 4500, 8, "chain", 1, 32),
    (F32, 64, 2, 1, 128, 2, 4500, 9, "tree", 1, 32),
    (BF, 128, 8, 2, 8, 33, 1200, 32, "tree", 1, 64),
    (BF, 128, 4, 8, 64, 9, 2600, 40, "dag", 2, 64),
    (BF, 64, 8, 2, 8, 40, 1200, 32, "chain", 1, 64),
    (F32, 128, 8, 2, 8, 9, 1200, 64, "chain", 1, 64),
    (F32, 64, 8, 2, 64, 33, 1200, 32, "shared", 1, 64),
    (BF, 128, 8, 8, 8, 9, 1200, 64, "chain", 1, 128),
    (BF, 128, 8, 2, 64, 24, 2600, 64, "dag", 2, 128),
    (BF, 64, 2, 8, 8, 40, 1200, 100, "tree", 1, 128),
    (F32, 128, 8, 8, 8, 16, 700, 64, "tree", 1, 128),
]


def ragged(case):
    """A long and a half-long sequence, the others short."""
    dt, D, Hkv, G, page, B, longest, n, mask, splits, rows = CASES[case]
    rng = np.random.default_rng(900 + case)
    lens = [longest, longest // 2 + 3] + [int(x) for x in rng.integers(0, 70, B - 2)]
    nodes = [n, n - 1] + [int(x) for x in rng.integers(0, n + 1, B - 2)]
    cache, q, words, see, lens, nodes = tree_case((dt, D, Hkv, G, page, lens, n, nodes, mask, 0), 900 + 10 * case)
    # page 0, which stands in for pages that are missing, holds what no output may show
    odd = torch.full_like(cache.k_pages[:1], float("nan"))
    cache = skv.PagedKV(torch.cat([odd, cache.k_pages]), torch.cat([odd.fill_(float("inf")), cache.v_pages]),
                        cache.block_table + 1)
    return cache, q, words, see, lens, nodes


def lose_pages(cache, lens, nodes):
    """Table entries out of range, at both ends and in the middle."""
    page, B = cache.k_pages.shape[2], len(lens)
    last = [(lens[b] + nodes[b] - 1) // page for b in range(B)]
    bad = [-1, 2 ** 31 - 1, cache.k_pages.shape[0], -2 ** 31]
    tile = 32 * (last[0] * page // 64)  # a tile in the middle of sequence 0
    for i, at in enumerate([0, tile // page, (tile + 24) // page, last[0] * 3 // 4, last[0] - 1, last[0]]):
        cache.block_table[0, at] = bad[i % 4]
    cache.block_table[1, last[1] // 3] = cache.block_table[1, last[1]] = -7
    for b in range(2, B, 3):
        cache.block_table[b, max(last[b], 0)] = bad[b % 4]
    return tile, last


@pytest.mark.parametrize("case", range(len(CASES)))
def test_long_caches(case):
    dt, D, Hkv, G, page, B, longest, n, mask, splits, rows = CASES[case]
    cache, q, words, see, lens, nodes = ragged(case)
    out, guard = guarded(q.shape, dt, DEV)
    run_tree(cache, q, words, lens, nodes, n, splits, out)
    guard("tree out")
    # blocks of the rows meant, with more than sixteen steps
    on_gpu, count, ws = i32(lens), i32(nodes), torch.empty(1 << 28, dtype=torch.uint8, device=DEV)
    again = torch.full_like(out, float("nan"))
    first = launches(lambda: skv.speechkv_tree_attn(q, cache, on_gpu, longest, again, tree_mask=words, num_nodes=count,
                                                    num_splits=splits, workspace=ws))[0]
    units = B * Hkv * splits
    assert first == ((units if units < 32 else (units + 7) // 8 * 8) * -(-n * G // rows), 256)
    assert -(-(longest + n) // 32) // splits // (128 // rows) > 16
    check_tree(out, cache, q, see, lens, nodes, f"case {case}")


@pytest.mark.parametrize("case", range(len(CASES)))
def test_long_caches_with_missing_pages(case):
    dt, D, Hkv, G, page, B, longest, n, mask, splits, rows = CASES[case]
    cache, q, words, see, lens, nodes = ragged(case)
    tile, last = lose_pages(cache, lens, nodes)
    out, guard = guarded(q.shape, dt, DEV)
    run_tree(cache, q, words, lens, nodes, n, splits, out)
    guard("tree out")
    check_tree(out, cache, q, see, lens, nodes, f"case {case}")
    # an infinite value between the two missing pages of that tile (pages of 8
    # rows), else behind a missing page of sequence 1
    slot = tile + 9 if page == 8 else (last[1] // 3 + 1) * page
    b = 0 if page == 8 else 1
    pg, row = ref.slot_row(cache.block_table.cpu().numpy(), b, slot, page, cache.v_pages.shape[0])
    cache.v_pages[pg, :, row, 5] = 0.0
    zero = run_tree(cache, q, words, lens, nodes, n, splits)
    cache.v_pages[pg, :, row, 5] = float("-inf")
    far = run_tree(cache, q, words, lens, nodes, n, splits)
    assert bool(torch.isneginf(far[b, :nodes[b], :, 5]).all())
    far[b, :nodes[b], :, 5] = zero[b, :nodes[b], :, 5]
    assert torch.equal(far.nan_to_num(7.0), zero.nan_to_num(7.0))


@pytest.mark.parametrize("missing", [False, True])
@pytest.mark.parametrize("case", range(len(CASES)))
def test_every_key_counts_once(case, missing):
    """Zero queries weigh all keys alike, and every key's value is 1 in one
    random element: the outputs count the keys of each element.  The counts are
    small (35 of 4500 keys), so one key too many or too few shows.  Sums and
    weights are whole numbers, exact in fp32; the division is off by 2 u and the
    output by one rounding."""
    dt, D, Hkv, G, page, B, longest, n, mask, splits, rows = CASES[case]
    cache, q, words, see, lens, nodes = ragged(case)
    if missing:
        lose_pages(cache, lens, nodes)
    gen = torch.Generator().manual_seed(case)
    one = torch.randint(D, cache.v_pages.shape[:3], generator=gen)
    cache.v_pages[1:] = torch.nn.functional.one_hot(one, D)[1:].to(DEV, dt)
    out = run_tree(cache, torch.zeros_like(q), words, lens, nodes, n, splits).to("cpu", torch.float64).numpy()
    table, one = cache.block_table.cpu().numpy(), one.numpy()
    for b in range(B):
        where = [ref.slot_row(table, b, c, page, one.shape[0]) for c in range(lens[b] + nodes[b])]
        cached = [w for w in where[:lens[b]] if w]
        for g in range(Hkv):
            base = np.bincount([one[p, g, r] for p, r in cached], minlength=D)
            for i in range(nodes[b]):
                count = base.copy()
                for j in range(nodes[b]):
                    if where[lens[b] + j] and see(b, i, j):
                        p, r = where[lens[b] + j]
                        count[one[p, g, r]] += 1
                want = count / max(count.sum(), 1)
                err = np.abs(out[b, i, g * G:(g + 1) * G] - want)
                assert np.all(err <= (ref.HALF[dt] + 2 * ref.U) * (1 + 1e-6) * want), (b, g, i)


@pytest.mark.parametrize("case", range(len(CASES)))
def test_every_row_finds_its_key(case):
    """Keys of random signs and queries that are eight times one of them: a row's
    output is that key's value, among them the keys on both sides of every
    sixteenth step of a stream."""
    dt, D, Hkv, G, page, B, longest, n, mask, splits, rows = CASES[case]
    cache, q, words, see, lens, nodes = ragged(case)
    signs = torch.randint(2, cache.k_pages[1:].shape, generator=torch.Generator().manual_seed(case))
    cache.k_pages[1:] = (signs * 2 - 1).to(DEV, dt)
    rng = np.random.default_rng(case)
    table, edge = cache.block_table.cpu().numpy(), 16 * (128 // rows) * 32
    for b in range(B):
        for i in range(nodes[b]):
            for h in range(Hkv * G):
                if lens[b] == 0:
                    continue
                slot = int(rng.integers(lens[b]))
                if b == 0 and h % 2:  # near a multiple of sixteen steps
                    slot = min(max(0, edge * int(rng.integers(1, lens[0] // edge + 1)) + int(rng.integers(-160, 160))),
                               lens[0] - 1)
                p, r = ref.slot_row(table, b, slot, page, cache.k_pages.shape[0])
                q[b, i, h] = 8 * cache.k_pages[p, h // G, r]
    out = run_tree(cache, q, words, lens, nodes, n, splits)
    check_tree(out, cache, q, see, lens, nodes, f"case {case}")
