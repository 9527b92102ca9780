"""Entry weights of prompts by blocks of two stretches of keys, with row tiles that
go through a wave's buffers more than once, on the GPU against the 64-bit form.

Bound.  A weight is off as tests/shared_ref.py derives it: its exponent by (D + 4) U
of scale sum |q k|, 3 U of |z| + |l| and 2 U.  Of one key a lane adds a row of every
eighth row tile; 16 lanes add up in 4 steps, the 8 waves in turn, and what the entry
had comes last: ceil(tiles / 8) + 4 + 8 + 1 roundings of a sum at most.
"""
import pytest
import torch

from gpu_case import guarded
from paper_2607_06827_amd import inputs
from paper_2607_06827_amd import speechkv as skv
from shared_ref import U
from test_gpu_draft import i32, make_cache
from test_gpu_shared import poison
from weights_cases import F32, TWO_STRETCHES, row_tiles

pytestmark = [pytest.mark.gpu,
              pytest.mark.skipif(not torch.cuda.is_available(), reason="needs a GPU")]

DEV = "cuda"


def seen_by(how, lens, n, seed):
    """int64 [B, n]: how many entries each row sees, before clipping."""
    g = torch.Generator().manual_seed(seed)
    rows = []
    for L in lens:
        if how == "last":
            rows.append(torch.arange(n) + L - (n - 1))
        else:
            r = torch.randint(-2, L + 3, (n,), generator=g)
            rows.append(r.sort().values if how == "rising" else r)
    return torch.stack(rows)


@pytest.mark.parametrize("case", range(len(TWO_STRETCHES)))
def test_two_stretches(case):
    dt, D, Hq, Hkv, page, lens, n, how = TWO_STRETCHES[case]
    B, G, most, scale = len(lens), Hq // Hkv, max(lens), D ** -0.5
    cache = make_cache(B, most, Hkv, D, dt, page, seed=1000 + case)
    poison(cache, lens)
    q = inputs.normal((B, n + 3, Hq + 1, D), 1100 + case, dtype=dt).to(DEV)[:, 2:n + 2, 1:]
    seen = seen_by(how, lens, n, case)
    table = cache.block_table.long()
    lse = torch.full((Hq, B, n), float("-inf"), device=DEV).transpose(0, 1)
    had = torch.rand(B, Hkv, most + 5, device=DEV)
    parts = {}
    for b, L in enumerate(lens):
        s = torch.arange(L, device=DEV)
        keys = cache.k_pages[table[b, s // page], :, s % page].double()  # [L, Hkv, D]
        use = s < seen[b].clamp(0, L).to(DEV)[:, None]  # [n, L]
        for h in range(Hq):
            k = keys[:, h // G]
            z = torch.matmul(q[b, :, h].double(), k.T.contiguous()) * scale
            if L:
                lse[b, h] = torch.where(use, z, float("-inf")).logsumexp(1).float()
            size = torch.matmul(q[b, :, h].double().abs(), k.abs().T.contiguous()) * scale
            l = lse[b, h].double()
            used = use & ~torch.isneginf(l)[:, None]
            l = torch.where(torch.isneginf(l), 0.0, l)[:, None]
            p = torch.where(used, torch.exp(torch.where(used, z - l, 0.0)), 0.0)
            off = p * ((D + 4) * U * size + 3 * U * (z.abs() + l.abs()) + 2 * U)
            # row i of head h is in tile (i G + h % G) / 16
            tile = (torch.arange(n, device=DEV) * G + h % G) // 16
            sums = torch.zeros(row_tiles(TWO_STRETCHES[case]), L, dtype=torch.float64, device=DEV).index_add_(0, tile, p)
            a = parts.setdefault((b, h // G), [0.0, 0.0, 0.0])
            parts[b, h // G] = [a[0] + p.sum(0), a[1] + off.sum(0), a[2] + sums]

    results = []
    for visible in (i32(seen.tolist()), None)[:2 if how == "last" else 1]:
        out, behind = guarded((B, Hkv, most + 5), F32, DEV, fill=-3.0)
        skv.speechkv_attn_weights(q, lse, cache, i32(lens), most, out, weights=had, visible=visible)
        torch.cuda.synchronize()
        behind("weights")
        results.append(out)
    assert all(torch.equal(r, results[0]) for r in results)
    again = had.clone()
    skv.speechkv_attn_weights(q, lse, cache, i32(lens), most, again, weights=again, visible=i32(seen.tolist()))
    deep = -(-row_tiles(TWO_STRETCHES[case]) // 8) + 13
    tiles = told = 0
    for b, L in enumerate(lens):
        assert bool((results[0][b, :, L:] == -3.0).all()) and torch.equal(again[b, :, L:], had[b, :, L:])
        assert torch.equal(again[b, :, :L], results[0][b, :, :L])
        for g in range(Hkv):
            p, off, by_tile = parts[b, g]
            start = had[b, g, :L].double()
            bound = (off + deep * U * (p + start)) * (1 + 1e-6)
            got = results[0][b, g, :L].double()
            assert bool(((got - start - p).abs() <= bound).all()), (b, g, float(((got - start - p).abs() - bound).max()))
            # the bound tells: a row tile that is lost, or added twice, shows
            live = by_tile.amax(1) > 0 if L else torch.zeros(0, dtype=torch.bool)
            tiles += int(live.sum())
            told += int(((by_tile > 2 * bound).any(1) & live).sum()) if L else 0
    assert tiles and told == tiles, (told, tiles)
