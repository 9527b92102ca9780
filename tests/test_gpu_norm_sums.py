"""The sums over rows of speechkv_norm_rope_bwd (dgamma) against 64-bit ones, with
a bound small enough that a lost sequence, and nearly any lost token, shows.

Bound.  U = 2^-24.  A term t = g n of a row and head is off by e = |n| eg + 16 U |t|
(tests/norm_ref.py: n = r x by 15 U, the product by one, g by eg where it was turned
back).  The terms of one element are added in four steps, so a term goes through as
many roundings as the sum of their lengths:
 - a lane group adds the rows of its own one after the other: waves take steps of at
   most 8 tokens in turn, and a wave's 8 or 16 lane groups deal out the step's rows;
 - a block adds its 4 x 8 (head_dim 128) or 4 x 16 (64) lane groups in turn;
 - 128 threads add the blocks' sums, each every 128th;
 - and 7 steps of a tree add the threads.
A rounding is U of the partial sum, at most U of the sum of absolute terms.
"""
import numpy as np
import pytest
import torch

import norm_ref as ref
from draft_ref import f64
from gpu_case import guarded
from paper_2607_06827_amd import inputs
from paper_2607_06827_amd import speechkv as skv
from test_gpu_norm import CASES, DEV, F32, Inputs, gamma64

NORMED = [i for i, c in enumerate(CASES) if c[12]]
FULL = 8192  # waves that fill the chip


def roundings(tokens, heads, blocks, D):
    """Most roundings of a term of one element: `tokens` tokens of `heads` heads in
    `blocks` blocks."""
    groups = 64 // (D // 16)
    # rows of a lane group.  Few tokens (below FULL / 2 waves' steps): a step is a
    # token, `split` waves share it; many: a step has up to 8 tokens.
    split = min(-(-heads // groups), 1 + 8 * FULL // tokens) if tokens < FULL // 2 else 1
    step = 1
    while step < 8 and step * heads < 4 * groups and tokens // (2 * step) >= FULL:
        step *= 2
    turns = -(-(-(-tokens // step) * split) // (4 * blocks))
    rows = turns * -(-(step * heads) // (groups * split))
    return rows + 4 * groups + -(-blocks // 128) + 7


def blocks_of(tokens, heads, of_both, D):
    """Blocks of one kind of rows: what the waves take, and no more than its share of
    2048 and one."""
    groups = 64 // (D // 16)
    split = min(-(-heads // groups), 1 + 8 * FULL // tokens) if tokens < FULL // 2 else 1
    step = 1
    while step < 8 and step * heads < 4 * groups and tokens // (2 * step) >= FULL:
        step *= 2
    return min(-(-(-(-tokens // step) * split) // 4), 1 + FULL // 4 * heads // of_both)


def sums(x, src, gamma, dy):
    """Per sequence: sum of the terms, of their absolute values, of their errors, and
    the terms of each token, added over its heads."""
    out = []
    for b in range(x.B):
        n = x.n[b]
        if not n:
            out.append((np.zeros(x.D), np.zeros(x.D), np.zeros(x.D), np.zeros((0, x.D))))
            continue
        X, G = f64(src[b, :n]), f64(dy[b, :n])
        rot = x.rot_of(b)
        if rot is None:
            g, eg = G, np.zeros_like(G)
        else:
            g, size, err, stays = ref.turned(G, *rot, sign=-1.0)
            eg = (np.where(stays, 0.0, 7 * ref.U) + err) * size
        nx = X / np.sqrt((X * X).mean(-1, keepdims=True) + x.eps)
        t = g * nx
        e = np.abs(nx) * eg + 16 * ref.U * np.abs(t)
        out.append((t.sum((0, 1)), np.abs(t).sum((0, 1)), e.sum((0, 1)), t.sum(1)))
    return out


def expected(x, kind):
    """(dgamma, its bound, per sequence its part, its tokens' parts)."""
    src, gamma, dy = x.parts()[kind]
    per = sums(x, src, gamma64(gamma), dy)
    total, size, err = (sum(p[i] for p in per) for i in range(3))
    heads = (x.Hq, x.Hkv)
    blocks = blocks_of(x.B * x.S, heads[kind], sum(heads), x.D)
    deep = roundings(x.B * x.S, heads[kind], blocks, x.D)
    return total, (err + deep * ref.U * (size + err)) * (1 + 1e-6), per


@pytest.mark.gpu
@pytest.mark.skipif(not torch.cuda.is_available(), reason="needs a GPU")
@pytest.mark.parametrize("case", NORMED)
def test_dgamma(case):
    x = Inputs(case, seed=1)
    outs = [torch.full((x.B, x.S, h, x.D), -7.0, dtype=x.dt, device=DEV) for h in (x.Hq, x.Hkv)]
    got = [guarded((x.D,), F32, DEV) for _ in range(2)]
    ws, behind = guarded((skv.speechkv_norm_rope_bwd_workspace_bytes(x.B, x.S, x.Hq, x.Hkv, x.D) // 4,), F32, DEV)
    skv.speechkv_norm_rope_bwd(x.q, x.k, x.dq_out, x.dk_out, *outs, row_len=x.row_len, dgamma_q=got[0][0],
                               dgamma_k=got[1][0], workspace=ws, **x.common())
    torch.cuda.synchronize()
    behind("workspace")
    for kind in (0, 1):
        got[kind][1]("dgamma")
        total, bound, per = expected(x, kind)
        off = np.abs(f64(got[kind][0]) - total)
        assert np.all(off <= bound), (kind, np.max(off / bound))
        # the bound tells: zeros do not pass, nor does a sum without one sequence,
        # nor one without any single token (of nearly all)
        if sum(x.n):
            assert np.any(np.abs(total) > bound), kind
        seen = lost = 0
        for part, _, _, tokens in per:
            if len(tokens):
                assert np.any(np.abs(part) > 2 * bound), kind
                seen += len(tokens)
                lost += int((np.abs(tokens) > 2 * bound).any(1).sum())
        assert lost >= 0.99 * seen, (kind, lost, seen)


@pytest.mark.gpu
@pytest.mark.skipif(not torch.cuda.is_available(), reason="needs a GPU")
def test_blocks_are_those_of_the_bound():
    """The sums in the workspace: as many as the bound counts blocks."""
    for case in NORMED:
        x = Inputs(case, seed=1)
        outs = [torch.empty((x.B, x.S, h, x.D), dtype=x.dt, device=DEV) for h in (x.Hq, x.Hkv)]
        room = skv.speechkv_norm_rope_bwd_workspace_bytes(x.B, x.S, x.Hq, x.Hkv, x.D) // 4
        ws = torch.full((room // x.D, x.D), float("nan"), device=DEV)
        dg = torch.empty(2, x.D, device=DEV)
        skv.speechkv_norm_rope_bwd(x.q, x.k, x.dq_out, x.dk_out, *outs, row_len=x.row_len, dgamma_q=dg[0], dgamma_k=dg[1],
                                   workspace=ws, **x.common())
        blocks = sum(blocks_of(x.B * x.S, h, x.Hq + x.Hkv, x.D) for h in (x.Hq, x.Hkv))
        assert int(torch.isfinite(ws).all(1).sum()) == blocks and bool(torch.isfinite(ws[:blocks]).all()), case
