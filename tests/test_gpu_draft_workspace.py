"""speechkv_tree_attn with less workspace than its best split count wants, on
the GPU against the 64-bit form: right values, nothing written behind it."""
import pytest
import torch

from gpu_case import guarded
from paper_2607_06827_amd import speechkv as skv
from test_gpu_draft import BF, DEV, F32, check_tree, i32, run_tree, tree_case

pytestmark = [pytest.mark.gpu,
              pytest.mark.skipif(not torch.cuda.is_available(), reason="needs a GPU")]


@pytest.mark.parametrize("dt", [BF, F32])
def test_any_workspace_gives_the_same_attention(dt):
    n, lens = 12, [900, 870]
    cache, q, words, see, lens, nodes = tree_case((dt, 128, 2, 2, 16, lens, n, [12, 9], "tree", 0), 21)
    best = skv.speechkv_tree_num_splits(2, n, 4, 2, 128, dt, 900)
    assert best >= 4
    a_split = 2 * n * 4 * 130 * 4
    for room in (0, 16, 2 * a_split - 16, 2 * a_split, 3 * a_split, best * a_split, 40 * a_split):
        out, rows = guarded(q.shape, dt, DEV)
        ws, behind = guarded((max(room, 16) // 4,), F32, DEV)
        skv.speechkv_tree_attn(q, cache, i32(lens), 900, out, tree_mask=words, num_nodes=i32(nodes),
                               workspace=ws if room else None)
        rows(f"out, {room} bytes")
        behind(f"workspace, {room} bytes")
        check_tree(out, cache, q, see, lens, nodes, f"{room} bytes")
        untouched = bool(torch.isnan(ws).all())
        assert untouched == (room < 2 * a_split), room
        # the bits are those of the split count that fits
        fits = max(s for s in (1, 2, 3, best) if s == 1 or s * a_split <= room)
        if fits in (1, best):
            given = run_tree(cache, q, words, lens, nodes, n, fits)
            assert torch.equal(given.nan_to_num(7.0), out.nan_to_num(7.0)), room
