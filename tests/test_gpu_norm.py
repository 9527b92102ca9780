"""Per-head norms with rotation on the GPU: forward, gradients and the append,
against plain 64-bit forms (tests/norm_ref.py, which derives the bounds)."""
import numpy as np
import pytest
import torch

import norm_ref as ref
from draft_ref import HALF, f64
from gpu_case import guarded
from paper_2607_06827_amd import inputs
from paper_2607_06827_amd import speechkv as skv
from test_gpu_draft import i32, make_cache, rows_of

pytestmark = [pytest.mark.gpu,
              pytest.mark.skipif(not torch.cuda.is_available(), reason="needs a GPU")]

DEV = "cuda"
BF, F32 = torch.bfloat16, torch.float32

CASES = [
    # dtype, D, Hq, Hkv, B, S, rot, pairs, axes, counts, strides, far, norm, gammas
    (BF, 128, 16, 8, 1, 1, 128, False, 1, None, "fused", 0, True, True),
    (BF, 128, 16, 8, 3, 7, 128, False, 3, [7, 3, 0], "fused", 0, True, True),
    (BF, 64, 4, 4, 2, 33, 32, True, 2, None, "dense", 10 ** 6, True, True),
    (F32, 64, 8, 1, 2, 5, 16, True, 1, [5, 1], "fused", 0, True, False),
    (F32, 128, 8, 2, 4, 65, 128, False, 2, [65, 64, 2, 1], "wide", 40000, True, True),
    (F32, 128, 4, 2, 1, 300, 96, False, 1, None, "dense", 2 ** 31 - 400, True, True),
    (BF, 64, 3, 2, 2, 9, 0, False, 1, [4, 9], "wide", 0, True, True),
    (BF, 128, 2, 2, 65, 2, 48, True, 3, [i % 3 for i in range(65)], "fused", 100, True, True),
    (BF, 128, 5, 3, 2, 11, 64, False, 2, None, "fused", -70000, False, False),
    (F32, 64, 1, 1, 2, 3, 64, False, 16, None, "dense", 5, False, False),
    (BF, 64, 64, 8, 5, 301, 64, False, 3, [301, 0, 17, 300, 1], "fused", 1000, True, True),
    # many tokens: two and eight of them a step
    (F32, 128, 1, 1, 9, 2000, 128, True, 1, None, "fused", 7, True, True),
    (BF, 64, 2, 1, 33, 4000, 32, False, 2, [4000 - 119 * i for i in range(33)], "dense", 0, True, True),
]


class Inputs:
    def __init__(self, case, seed=0):
        (self.dt, self.D, self.Hq, self.Hkv, self.B, self.S, self.rot, self.pairs, self.axes, self.counts, strides,
         far, self.norm, gammas) = CASES[case]
        B, S, D, H = self.B, self.S, self.D, self.Hq + 2 * self.Hkv
        self.n = self.counts or [S] * B

        def views(seed):
            if strides == "fused":
                x = inputs.normal((B, S, H, D), seed, dtype=self.dt).to(DEV)
            elif strides == "wide":  # heads outermost, rows apart
                x = inputs.normal((H, B, S + 2, D + 16), seed, dtype=self.dt).to(DEV).permute(1, 2, 0, 3)[:, 1:S + 1, :, :D]
            else:
                return tuple(inputs.normal((B, S, h, D), seed + i, dtype=self.dt).to(DEV)
                             for i, h in enumerate((self.Hq, self.Hkv, self.Hkv)))
            return x[:, :, :self.Hq], x[:, :, self.Hq:self.Hq + self.Hkv], x[:, :, self.Hq + self.Hkv:]

        self.q, self.k, self.v = views(10 * seed + 1)
        self.dq_out, self.dk_out, _ = views(10 * seed + 5)
        for b in range(B):  # rows that a sequence does not have are never used
            for x in (self.q, self.k, self.v, self.dq_out, self.dk_out):
                x[b, self.n[b]:] = float("nan")
        pos = torch.arange(S)[None, None] + far + 3 * torch.arange(B)[None, :, None] + 7 * torch.arange(self.axes)[:, None, None]
        self.pos = pos.to(torch.int32)
        half = self.rot // 2
        self.inv = (1e4 ** (-torch.arange(0, self.rot, 2, dtype=torch.float64) / max(self.rot, 1))).float()
        self.axis = torch.arange(half, dtype=torch.int32) % self.axes
        self.gq, self.gk = ((1 + 0.3 * inputs.normal((D,), 77 + i, dtype=F32)).to(DEV) if gammas else None for i in (0, 1))
        self.eps = 1e-6 if self.norm else None
        self.rope = None
        if self.rot:
            self.rope = skv.Rope(self.pos.to(DEV) if self.axes > 1 else self.pos[0].to(DEV), self.inv.to(DEV),
                                 self.axis.to(DEV) if self.axes > 1 else None,
                                 skv.ROPE_PAIRS if self.pairs else skv.ROPE_HALVES)
        self.row_len = None if self.counts is None else i32(self.counts)

    def rot_of(self, b):
        if not self.rot:
            return None
        return self.pos[:, b, :self.n[b]].numpy(), self.inv.double().numpy(), self.axis.numpy(), self.pairs

    def common(self):
        return dict(gamma_q=self.gq, gamma_k=self.gk, rope=self.rope, normalise=self.norm)

    def parts(self):
        return ((self.q, self.gq, self.dq_out), (self.k, self.gk, self.dk_out))


def gamma64(g):
    return None if g is None else f64(g)


def check(got, want, bound, what):
    off = np.abs(f64(got) - want) - bound
    assert np.all(off <= 0), (what, np.max(off), np.unravel_index(np.argmax(off), off.shape))


@pytest.mark.parametrize("case", range(len(CASES)))
def test_norm_rope(case):
    x = Inputs(case)
    outs = [guarded((x.B, x.S, h, x.D), x.dt, DEV, fill=-7.0) for h in (x.Hq, x.Hkv)]
    skv.speechkv_norm_rope(x.q, x.k, outs[0][0], outs[1][0], row_len=x.row_len, **x.common())
    torch.cuda.synchronize()
    for (src, gamma, _), (out, guard) in zip(x.parts(), outs):
        guard("norm out")
        for b in range(x.B):
            n = x.n[b]
            if n:
                want, bound = ref.forward(f64(src[b, :n]), gamma64(gamma), x.eps, x.rot_of(b), HALF[x.dt])
                check(out[b, :n], want, bound, b)
            assert bool((out[b, n:] == -7.0).all())


@pytest.mark.parametrize("case", range(len(CASES)))
def test_norm_rope_gradients(case):
    x = Inputs(case, seed=1)
    outs = [guarded((x.B, x.S, h, x.D), x.dt, DEV, fill=-7.0) for h in (x.Hq, x.Hkv)]
    sums = [guarded((x.D,), F32, DEV) for _ in range(2)] if x.norm else [(None, None)] * 2
    need = skv.speechkv_norm_rope_bwd_workspace_bytes(x.B, x.S, x.Hq, x.Hkv, x.D)
    ws, ws_guard = guarded((need // 4,), F32, DEV)
    skv.speechkv_norm_rope_bwd(x.q, x.k, x.dq_out, x.dk_out, outs[0][0], outs[1][0], row_len=x.row_len,
                               dgamma_q=sums[0][0], dgamma_k=sums[1][0], workspace=ws, **x.common())
    torch.cuda.synchronize()
    ws_guard("workspace")
    for (src, gamma, dy), (out, guard), (dgamma, sum_guard) in zip(x.parts(), outs, sums):
        guard("gradient")
        total, total_bound, terms = np.zeros(x.D), np.zeros(x.D), 0.0
        for b in range(x.B):
            n = x.n[b]
            assert bool((out[b, n:] == -7.0).all())
            if not n:
                continue
            dx, bound, dg, bg = ref.backward(f64(src[b, :n]), f64(dy[b, :n]), gamma64(gamma), x.eps, x.rot_of(b),
                                             HALF[x.dt])
            check(out[b, :n], dx, bound, b)
            if x.norm:
                total += dg
                total_bound += bg + x.B * ref.U * np.abs(dg)
        if x.norm:
            sum_guard("dgamma")
            # (each sequence's bound counts its own terms; adding the sequences to
            # one sum takes as many roundings again as there are rows in all)
            rows = sum(x.n) * src.shape[2]
            total_bound = total_bound * (1 + rows / max(1, min(n for n in x.n if n) * src.shape[2]))
            check(dgamma, total, total_bound, "dgamma")


def test_in_place_and_beside_each_other():
    """Outputs that are their inputs, inside one projection's output: the values
    beside them stay."""
    x = Inputs(1)
    qkv = x.q._base if x.q._base is not None else x.q
    q_out, k_out = torch.empty_like(x.q.contiguous()), torch.empty_like(x.k.contiguous())
    skv.speechkv_norm_rope(x.q, x.k, q_out, k_out, row_len=x.row_len, **x.common())
    v = x.v.clone()
    grads = [torch.empty_like(t.contiguous()) for t in (x.q, x.k)]
    skv.speechkv_norm_rope_bwd(x.q, x.k, x.dq_out, x.dk_out, *grads, row_len=x.row_len, **x.common())
    skv.speechkv_norm_rope_bwd(x.q, x.k, x.dq_out, x.dk_out, x.dq_out, x.dk_out, row_len=x.row_len, **x.common())
    skv.speechkv_norm_rope(x.q, x.k, x.q, x.k, row_len=x.row_len, **x.common())
    assert qkv.is_cuda
    for b, n in enumerate(x.n):
        assert torch.equal(x.q[b, :n], q_out[b, :n]) and torch.equal(x.k[b, :n], k_out[b, :n])
        assert torch.equal(x.v[b, :n], v[b, :n])
        assert torch.equal(x.dq_out[b, :n], grads[0][b, :n]) and torch.equal(x.dk_out[b, :n], grads[1][b, :n])


def test_more_heads_than_waves_share():
    # a row gives the same bits in a call of all heads as in one of a few
    S, H, D = 4095, 160, 128
    q, dy = (inputs.normal((1, S, H, D), i, dtype=BF).to(DEV) for i in (1, 2))
    gamma = (1 + 0.3 * inputs.normal((D,), 3, dtype=F32)).to(DEV)
    rope = skv.Rope(torch.arange(S, dtype=torch.int32, device=DEV)[None],
                    torch.logspace(0, -4, D // 2, dtype=F32, device=DEV))
    out, dq, some, dsome = (torch.full_like(q, -7.0) for _ in range(4))
    skv.speechkv_norm_rope(q, None, out, None, gamma_q=gamma, rope=rope)
    skv.speechkv_norm_rope_bwd(q, None, dy, None, dq, None, gamma_q=gamma, rope=rope)
    for h in range(0, H, 40):
        at = (slice(None), slice(None), slice(h, h + 40))
        skv.speechkv_norm_rope(q[at], None, some[at], None, gamma_q=gamma, rope=rope)
        skv.speechkv_norm_rope_bwd(q[at], None, dy[at], None, dsome[at], None, gamma_q=gamma, rope=rope)
    assert torch.equal(out, some) and torch.equal(dq, dsome)
    assert bool((out[0, 0, :, 5] != -7.0).all())


@pytest.mark.parametrize("which", ["q", "k"])
def test_one_of_the_two(which):
    x = Inputs(4)
    both = [torch.zeros_like(t.contiguous()) for t in (x.q, x.k)]
    skv.speechkv_norm_rope(x.q, x.k, *both, row_len=x.row_len, **x.common())
    one = torch.zeros_like(both[which == "k"])
    args = (x.q, None, one, None) if which == "q" else (None, x.k, None, one)
    skv.speechkv_norm_rope(*args, row_len=x.row_len, **x.common())
    assert torch.equal(one, both[which == "k"])
    need = skv.speechkv_norm_rope_bwd_workspace_bytes(x.B, x.S, x.Hq, x.Hkv, x.D)
    ws = torch.empty(need, dtype=torch.uint8, device=DEV)
    grads, dg = [torch.zeros_like(t) for t in both], [torch.zeros(x.D, device=DEV) for _ in range(4)]
    skv.speechkv_norm_rope_bwd(x.q, x.k, x.dq_out, x.dk_out, *grads, row_len=x.row_len, dgamma_q=dg[0], dgamma_k=dg[1],
                               workspace=ws, **x.common())
    i = which == "k"
    src, dy = (x.k, x.dk_out) if i else (x.q, x.dq_out)
    one = torch.zeros_like(grads[i])
    none = dict(row_len=x.row_len, workspace=ws, **x.common())
    if i:
        skv.speechkv_norm_rope_bwd(None, src, None, dy, None, one, dgamma_k=dg[3], **none)
    else:
        skv.speechkv_norm_rope_bwd(src, None, dy, None, one, None, dgamma_q=dg[3], **none)
    assert torch.equal(one, grads[i]) and torch.equal(dg[3], dg[i])


def test_plain_rows_are_copied_bitwise():
    """No norm and no rotation; NaN payloads and infinities stay."""
    bits = torch.randint(-2 ** 15, 2 ** 15, (2, 5, 3, 64), dtype=torch.int16, device=DEV)
    x, out = bits.view(BF), torch.zeros(2, 5, 3, 64, dtype=BF, device=DEV)
    skv.speechkv_norm_rope(x, None, out, None, normalise=False)
    assert torch.equal(out.view(torch.int16), bits)


@pytest.mark.parametrize("dt", [BF, F32])
def test_values_at_the_borders(dt):
    """Rows of zeros give zeros, infinite and NaN rows stay their own trouble,
    tiny rows are normed by eps, huge ones count as infinitely long."""
    x = inputs.normal((1, 8, 2, 128), 3, dtype=dt).to(DEV)
    x[0, 1] = 0.0
    x[0, 2, 0, 5] = float("inf")
    x[0, 3, 1, 7] = float("nan")
    x[0, 4] *= 1e-30
    x[0, 5] = 1e25
    out = torch.empty_like(x)
    skv.speechkv_norm_rope(x, None, out, None, eps=1e-6)
    assert bool((out[0, 1] == 0).all()) and bool((out[0, 5] == 0).all())
    assert bool(torch.isnan(out[0, 2, 0, 5])) and bool(torch.isnan(out[0, 3, 1]).all())
    for rows in ((0, slice(None)), (2, 1), (3, 0), (4, slice(None)), (6, slice(None)), (7, slice(None))):
        src = f64(x[0][rows]).reshape(1, -1, 128)
        want, bound = ref.forward(src, None, 1e-6, None, HALF[dt])
        # (results below the normal range of the element type may round to 0)
        check(out[0][rows].reshape(1, -1, 128), want, bound + 2.0 ** -126, rows)


def test_axis_numbers_outside_the_axes_count_as_the_nearest():
    x = inputs.normal((1, 4, 2, 64), 3, dtype=F32).to(DEV)
    pos = torch.tensor([[[3, 5, 7, 9]], [[100, 200, 300, 400]]], dtype=torch.int32, device=DEV)
    inv = torch.rand(8, device=DEV)
    outs = []
    for axis in ([-5, 0, 1, 9, 0, 1, 2 ** 31 - 1, -2 ** 31], [0, 0, 1, 1, 0, 1, 1, 0]):
        out = torch.empty_like(x)
        skv.speechkv_norm_rope(x, None, out, None, rope=skv.Rope(pos, inv, i32(axis)))
        outs.append(out)
    assert torch.equal(*outs)


@pytest.mark.parametrize("case", range(len(CASES)))
def test_append(case):
    x = Inputs(case, seed=2)
    lens = [(5 * b) % 37 for b in range(x.B)]
    page = [8, 16, 64][case % 3]
    cache = make_cache(x.B, max(lens) + x.S, x.Hkv, x.D, x.dt, page, seed=300 + case)
    k0, v0 = cache.k_pages.clone(), cache.v_pages.clone()
    q_out, guard = guarded((x.B, x.S, x.Hq, x.D), x.dt, DEV, fill=-7.0)
    dense = [torch.full((x.B, x.S, h, x.D), -7.0, dtype=x.dt, device=DEV) for h in (x.Hq, x.Hkv)]
    skv.speechkv_norm_rope(x.q, x.k, *dense, row_len=x.row_len, **x.common())
    out_len = i32([-1] * x.B)
    skv.speechkv_norm_append_kv(x.q, x.k, x.v, cache, i32(lens), q_out, new_len=x.row_len, cache_len_out=out_len,
                                **x.common())
    guard("append q_out")
    assert out_len.tolist() == [a + b for a, b in zip(lens, x.n)]
    assert torch.equal(q_out, dense[0])
    touched = torch.zeros(cache.k_pages.shape[0], page, dtype=torch.bool, device=DEV)
    for b in range(x.B):
        gk, gv = rows_of(cache, b, lens[b], x.n[b])
        assert torch.equal(gk, dense[1][b, :x.n[b]]) and torch.equal(gv, x.v[b, :x.n[b]])
        s = torch.arange(lens[b], lens[b] + x.n[b], device=DEV)
        touched[cache.block_table[b, s // page].long(), s % page] = True
    same = ~touched[:, None, :, None]
    assert torch.equal(torch.where(same, cache.k_pages, k0), k0) and torch.equal(torch.where(same, cache.v_pages, v0), v0)


def test_append_without_queries_and_without_pages():
    """Bad table entries, slots past the table and negative lengths: neither
    read nor written out of range; the other rows are stored."""
    B, S, Hkv, D, page = 4, 6, 2, 64, 8
    cache = make_cache(B, 16, Hkv, D, BF, page)
    cache.block_table[0, 0] = -1
    cache.block_table[1, 1] = cache.k_pages.shape[0]
    lens = [5, 5, 13, -4]
    k, v = (inputs.normal((B, S, Hkv, D), 20 + i, dtype=BF).to(DEV) for i in range(2))
    k0, v0, t = cache.k_pages.clone(), cache.v_pages.clone(), cache.block_table.tolist()
    out_len, dense = i32([0] * B), torch.empty_like(k)
    skv.speechkv_norm_rope(None, k, None, dense)
    skv.speechkv_norm_append_kv(None, k, v, cache, i32(lens), new_len=i32([6, 6, 99, 2]), cache_len_out=out_len)
    assert out_len.tolist() == [11, 11, 19, 2]
    for b in range(B):
        for i in range([6, 6, 6, 2][b]):
            slot = max(lens[b], 0) + i
            if slot < 16 and 0 <= t[b][slot // page] < k0.shape[0]:
                k0[t[b][slot // page], :, slot % page] = dense[b, i]
                v0[t[b][slot // page], :, slot % page] = v[b, i]
    assert torch.equal(cache.k_pages, k0) and torch.equal(cache.v_pages, v0)


def test_the_append_without_a_norm_is_the_rotating_append():
    x = Inputs(2)
    a, b = make_cache(2, 60, 4, 64, BF, seed=9), make_cache(2, 60, 4, 64, BF, seed=9)
    q1, q2 = torch.empty_like(x.q), torch.empty_like(x.q)
    lens, rope = i32([3, 20]), skv.Rope(x.pos[0].to(DEV), x.inv.to(DEV), None, skv.ROPE_PAIRS)
    skv.speechkv_norm_append_kv(x.q, x.k, x.v, a, lens, q1, rope=rope, normalise=False)
    skv.speechkv_append_kv(x.k, x.v, b, lens, x.pos[0].to(DEV), x.inv.to(DEV), skv.ROPE_PAIRS, q=x.q, q_out=q2)
    assert torch.equal(q1, q2) and torch.equal(a.k_pages, b.k_pages) and torch.equal(a.v_pages, b.v_pages)


def test_captured_and_on_another_stream():
    """Forward and gradients captured into a graph on a stream of their own and
    replayed over new inputs: the eager results, bit for bit."""
    x, y = Inputs(10), Inputs(10, seed=3)
    need = skv.speechkv_norm_rope_bwd_workspace_bytes(x.B, x.S, x.Hq, x.Hkv, x.D)

    def outputs():
        return [torch.zeros((x.B, x.S, h, x.D), dtype=x.dt, device=DEV) for h in (x.Hq, x.Hkv)] + \
            [torch.zeros((x.B, x.S, h, x.D), dtype=x.dt, device=DEV) for h in (x.Hq, x.Hkv)] + \
            [torch.zeros(x.D, device=DEV) for _ in range(2)] + [torch.empty(need, dtype=torch.uint8, device=DEV)]

    def step(o, stream=None):
        skv.speechkv_norm_rope(x.q, x.k, o[0], o[1], row_len=x.row_len, stream=stream, **x.common())
        skv.speechkv_norm_rope_bwd(x.q, x.k, x.dq_out, x.dk_out, o[2], o[3], row_len=x.row_len, dgamma_q=o[4],
                                   dgamma_k=o[5], workspace=o[6], stream=stream, **x.common())

    got = outputs()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(got)
    side = torch.cuda.Stream()
    for new in (x, y, x):
        for a, b in ((x.q, new.q), (x.k, new.k), (x.dq_out, new.dq_out), (x.dk_out, new.dk_out)):
            a.copy_(b.clone())
        want = outputs()
        torch.cuda.synchronize()
        step(want, stream=side)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got[:6], want[:6]))
