"""Views of one tensor in the calls of include/speechkv_norm.h, in every order
of its axes: what lies beside each other is accepted, what meets is refused."""
import random

import pytest
import torch

from paper_2607_06827_amd import inputs
from paper_2607_06827_amd import speechkv as skv
from test_abi import NO_GPU
from test_draft_abi import E_ALIAS, E_ARG, E_HIP, at
from test_norm_abi import append, bwd, fwd

ORDERS = ["bshd", "sbhd", "bhsd", "hbsd", "shbd", "hsbd"]  # outermost axis first


def parts(order, place, heads, B=2, S=3, D=64):
    """Views of neighbouring heads of one tensor whose axes lie in this order."""
    size, stride, step = dict(b=B, s=S, h=sum(heads), d=D), {}, 1
    for axis in reversed(order):
        stride[axis], step = step, step * size[axis]
    views, first = [], 0
    for h in heads:
        views.append(skv._Heads(place + first * stride["h"] * 2, stride["b"], stride["s"], stride["h"], h))
        first += h
    return views


@NO_GPU
@pytest.mark.parametrize("order", ORDERS)
@pytest.mark.parametrize("B,S", [(2, 3), (1, 5), (4, 1), (1, 1)])
def test_heads_of_one_tensor_lie_beside_each_other(order, B, S):
    q, k, v = parts(order, at(8), (4, 2, 2), B, S)
    size = dict(batch=B, rows=S, row_len=None, rope=None)
    assert fwd(q=q, k=k, q_out=q, k_out=k, **size) == E_HIP  # in place
    assert fwd(q=k, k=v, q_out=k, k_out=v, **size) == E_HIP
    oq, ok = parts(order, at(9), (4, 2), B, S)
    assert fwd(q=q, k=k, q_out=oq, k_out=ok, **size) == E_HIP  # out of one, into another
    dq, dk, _ = parts(order, at(10), (4, 2, 2), B, S)
    assert bwd(q=q, k=k, dyq=oq, dyk=ok, dq=dq, dk=dk, **size) == E_HIP
    assert bwd(q=q, k=k, dyq=dq, dyk=dk, dq=dq, dk=dk, **size) == E_HIP  # gradients in place
    assert append(q=q, k=k, v=v, q_out=q, **size) == E_HIP
    # a part shifted by a head meets its neighbour
    assert fwd(q=q, k=k, q_out=skv._Heads(k.data, q.stride_b, q.stride_s, q.stride_h, 4), k_out=ok, **size) == E_ALIAS


def rows(v, B, S, D):
    return {(v.data - at(8)) // 2 + b * v.stride_b + i * v.stride_s + h * v.stride_h + e
            for b in range(B) for i in range(S) for h in range(v.num_heads) for e in range(0, D, 8)}


@NO_GPU
def test_views_that_meet_are_refused():
    """Random views: a call that passes the checks has no element of an output in
    the other input or output."""
    rng, passed, met = random.Random(5), 0, 0
    D = 64
    for _ in range(30000):
        B, S, hq, hk = rng.randint(1, 3), rng.randint(1, 3), rng.randint(1, 3), rng.randint(1, 3)
        if rng.random() < 0.5:
            q, k = parts(rng.choice(ORDERS), at(8), (hq, hk), B, S)
            k.data += 2 * rng.choice([0, 0, 0, 8, 64, -64, 128])
            if rng.random() < 0.3:
                q.stride_s += 8 * rng.randint(0, 20)
                k.stride_s = q.stride_s
        else:
            stride = lambda: rng.choice([0, 8, 64, 64, 128, 192, 256, 384, 576, 768])  # noqa: E731
            sb, ss = stride(), stride()
            q = skv._Heads(at(8), sb, ss, stride(), hq)
            k = skv._Heads(at(8) + 16 * rng.randint(0, 100), *((sb, ss) if rng.random() < 0.8 else (stride(), stride())),
                           stride(), hk)
        st = fwd(q=q, k=k, q_out=q, k_out=k, batch=B, rows=S, row_len=None, rope=None)
        assert st in (E_HIP, E_ALIAS, E_ARG)
        a, b = rows(q, B, S, D), rows(k, B, S, D)
        lanes = {x + e for x in a for e in range(8)} & {x + e for x in b for e in range(8)}
        met += bool(lanes)
        if st == E_HIP:
            passed += 1
            assert not lanes, [(v.data, v.stride_b, v.stride_s, v.stride_h, v.num_heads) for v in (q, k)] + [B, S]
    assert passed > 3000 and met > 3000


@pytest.mark.gpu
@pytest.mark.skipif(not torch.cuda.is_available(), reason="needs a GPU")
@pytest.mark.parametrize("order", ORDERS)
@pytest.mark.parametrize("dt", [torch.bfloat16, torch.float32])
def test_fused_projections_in_every_order(order, dt):
    """Normed in place and gradients into one fused tensor: the bits of calls on
    dense tensors, and the values beside them stay."""
    B, S, Hq, Hkv, D = 3, 9, 4, 2, 64
    sizes = dict(b=B, s=S, h=Hq + 2 * Hkv, d=D)

    def fused(seed):
        x = inputs.normal(tuple(sizes[a] for a in order), seed, dtype=dt).cuda()
        return x, x.permute([order.index(a) for a in "bshd"])

    (_, x), (_, dy), (whole, dx) = fused(1), fused(2), fused(3)
    cut = lambda t: (t[:, :, :Hq], t[:, :, Hq:Hq + Hkv], t[:, :, Hq + Hkv:])  # noqa: E731
    q, k, v = cut(x)
    gamma = (1 + 0.3 * inputs.normal((2, D), 4, dtype=torch.float32)).cuda()
    rope = skv.Rope(torch.arange(B * S, dtype=torch.int32, device="cuda").view(B, S),
                    torch.logspace(0, -4, D // 2, device="cuda"))
    with_ = dict(gamma_q=gamma[0], gamma_k=gamma[1], rope=rope)
    want, dwant = ([t.contiguous().clone() for t in (q, k)] for _ in range(2))
    skv.speechkv_norm_rope(q.contiguous(), k.contiguous(), *want, **with_)
    skv.speechkv_norm_rope_bwd(q.contiguous(), k.contiguous(), *(t.contiguous() for t in cut(dy)[:2]), *dwant, **with_)
    beside = [v.clone(), cut(dx)[2].clone()]
    skv.speechkv_norm_rope_bwd(q, k, *cut(dy)[:2], *cut(dx)[:2], **with_)
    skv.speechkv_norm_rope(q, k, q, k, **with_)
    assert all(torch.equal(a, b) for a, b in zip((q, k), want))
    assert all(torch.equal(a, b) for a, b in zip(cut(dx)[:2], dwant))
    assert torch.equal(v, beside[0]) and torch.equal(cut(dx)[2], beside[1]) and whole.is_cuda
