"""The calls of include/speechkv_norm.h on the CPU: the header and the library
agree, invalid arguments are rejected before any HIP call, and the binding
refuses what it cannot pass on (no kernel is launched); the gradients that the
GPU tests compare with are those of the forward, by differences."""
import ctypes
import os
import re
import shutil
import subprocess

import numpy as np
import pytest
import torch

import norm_ref
from paper_2607_06827_amd import speechkv as skv
from test_abi import FAKE, NO_GPU, cache
from test_draft_abi import E_ALIAS, E_ARG, E_HIP, E_UNS, E_WS, at

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HEADER = os.path.join(ROOT, "include", "speechkv_norm.h")
lib = skv._lib
BF16, F32 = skv.DTYPE_BF16, skv.DTYPE_F32


def test_every_declared_symbol_is_exported():
    text = re.sub(r"/\*.*?\*/", "", open(HEADER).read(), flags=re.S)
    names = set(re.findall(r"\b(speechkv_[a-z0-9_]+)\s*\(", text))
    assert names == {"speechkv_norm_rope", "speechkv_norm_rope_bwd", "speechkv_norm_rope_bwd_workspace_bytes",
                     "speechkv_norm_append_kv"}
    for n in names:
        assert hasattr(lib, n) and callable(getattr(skv, n)), n


@pytest.mark.skipif(shutil.which("gcc") is None, reason="needs gcc")
def test_header_compiles_as_c_and_cxx(tmp_path):
    for std, cc, name in (("c11", "gcc", "x.c"), ("c++17", "g++", "x.cc")):
        src = tmp_path / name
        src.write_text('#include "speechkv_norm.h"\n#include <stdio.h>\n'
                       'int main(void) { printf("%zu %zu %zu", sizeof(speechkv_heads), sizeof(speechkv_head_norm), '
                       'sizeof(speechkv_rope)); return 0; }\n')
        exe = tmp_path / (name + ".exe")
        subprocess.run([cc, f"-std={std}", "-Wall", "-Wextra", "-Werror", "-pedantic",
                        f"-I{os.path.join(ROOT, 'include')}", str(src), "-o", str(exe)], check=True)
        sizes = subprocess.run([str(exe)], check=True, capture_output=True, text=True).stdout.split()
        assert [int(s) for s in sizes] == [ctypes.sizeof(x) for x in (skv._Heads, skv._HeadNorm, skv._Rope)]


def heads(i, h=4, B=2, S=3, D=64, sb=None, ss=None, sh=None, data=None):
    return skv._Heads(at(i) if data is None else data, S * h * D if sb is None else sb, h * D if ss is None else ss,
                      D if sh is None else sh, h)


def ref(x):
    return None if x is None else ctypes.byref(x)


def norm(gq=0, gk=0, eps=1e-6):
    return skv._HeadNorm(gq or None, gk or None, eps)


def rope(pos=at(40), inv=at(41), axis=at(42), axes=3, rot=64, layout=0):
    return skv._Rope(pos, inv, axis, axes, rot, layout)



def fwd(**kw):
    a = dict(q=heads(8), k=heads(9, 2), batch=2, rows=3, row_len=at(45), D=64, dt=BF16, norm=norm(at(43), at(44)),
             rope=rope(), q_out=heads(10), k_out=heads(11, 2))
    a.update(kw)
    return lib.speechkv_norm_rope(ref(a["q"]), ref(a["k"]), a["batch"], a["rows"], a["row_len"], a["D"], a["dt"],
                                  ref(a["norm"]), ref(a["rope"]), ref(a["q_out"]), ref(a["k_out"]), None)


def bwd(**kw):
    a = dict(q=heads(8), k=heads(9, 2), dyq=heads(12), dyk=heads(13, 2), batch=2, rows=3, row_len=at(45), D=64, dt=BF16,
             norm=norm(at(43), at(44)), rope=rope(), dq=heads(10), dk=heads(11, 2), dgq=at(46), dgk=at(47), ws=at(48),
             ws_bytes=1 << 20)
    a.update(kw)
    return lib.speechkv_norm_rope_bwd(ref(a["q"]), ref(a["k"]), ref(a["dyq"]), ref(a["dyk"]), a["batch"], a["rows"],
                                      a["row_len"], a["D"], a["dt"], ref(a["norm"]), ref(a["rope"]), ref(a["dq"]),
                                      ref(a["dk"]), a["dgq"], a["dgk"], a["ws"], a["ws_bytes"], None)


def append(c=None, **kw):
    a = dict(q=heads(8), k=heads(9, 2), v=heads(12, 2), batch=2, rows=3, row_len=at(45), norm=norm(at(43), at(44)),
             rope=rope(), clen=at(46), q_out=heads(10), out=at(47))
    a.update(kw)
    c = c or cache()
    return lib.speechkv_norm_append_kv(ref(a["q"]), ref(a["k"]), ref(a["v"]), a["batch"], a["rows"], a["row_len"],
                                       ref(a["norm"]), ref(a["rope"]), a["clen"], ctypes.byref(c), ref(a["q_out"]),
                                       a["out"], None)


INF, NAN = float("inf"), float("nan")
SHARED = [
    (dict(batch=0), E_ARG), (dict(batch=65536), E_ARG), (dict(rows=0), E_ARG), (dict(rows=1 << 24), E_UNS),
    (dict(row_len=at(45) + 2), E_ARG), (dict(norm=norm(eps=0.0)), E_ARG), (dict(norm=norm(eps=-1.0)), E_ARG),
    (dict(norm=norm(eps=NAN)), E_ARG), (dict(norm=norm(eps=INF)), E_ARG), (dict(norm=norm(eps=1e-40)), E_ARG),
    (dict(norm=norm(gq=at(43) + 8)), E_ARG), (dict(rope=rope(pos=None)), E_ARG), (dict(rope=rope(inv=None)), E_ARG),
    (dict(rope=rope(axes=0)), E_ARG), (dict(rope=rope(axes=17)), E_ARG), (dict(rope=rope(rot=0)), E_ARG),
    (dict(rope=rope(rot=24)), E_ARG), (dict(rope=rope(rot=80)), E_ARG), (dict(rope=rope(layout=2)), E_ARG),
    (dict(rope=rope(pos=at(40) + 1)), E_ARG), (dict(rope=rope(axis=at(42) + 2)), E_ARG),
    (dict(q=heads(8, data=at(8) + 8)), E_ARG), (dict(q=heads(8, sb=4)), E_ARG), (dict(q=heads(8, ss=-64)), E_ARG),
    (dict(q=heads(8, h=0)), E_ARG), (dict(q=heads(8, h=5)), E_ARG), (dict(q=heads(8, sb=1 << 61)), E_ARG),
    (dict(q=None), E_ARG), (dict(k=None), E_ARG), (dict(k=heads(9, 3)), E_ARG), (dict(k=skv._Heads()), E_ARG),
]
OUT = [(dict(q_out=None), E_ARG), (dict(q_out=heads(10, sh=0)), E_ARG), (dict(q_out=heads(10, ss=192)), E_ARG),
       (dict(q_out=heads(10, sb=0)), E_ARG), (dict(q_out=heads(10, sb=3 * 256 - 64)), E_ARG)]


@pytest.mark.parametrize("kw,code", SHARED + OUT + [
    (dict(D=32), E_UNS), (dict(dt=2), E_UNS), (dict(q=None, k=None, q_out=None, k_out=None), E_ARG)])
def test_forward_rejects(kw, code):
    assert fwd(**kw) == code


@pytest.mark.parametrize("kw,code", SHARED + [
    (dict(D=32), E_UNS), (dict(dt=2), E_UNS), (dict(dq=None), E_ARG), (dict(dyq=None), E_ARG), (dict(dyk=None), E_ARG),
    (dict(dq=heads(10, sh=0)), E_ARG), (dict(dk=heads(11, 4)), E_ARG), (dict(norm=None), E_ARG),
    (dict(q=None, dyq=None, dq=None), E_ARG),  # its dgamma is asked for
    (dict(ws=None), E_WS), (dict(ws=at(48) + 4), E_WS), (dict(ws_bytes=skv.speechkv_norm_rope_bwd_workspace_bytes(2, 3, 4, 2, 64) - 1), E_WS)])
def test_backward_rejects(kw, code):
    assert bwd(**kw) == code


@pytest.mark.parametrize("kw,code", SHARED + OUT + [
    (dict(v=None), E_ARG), (dict(clen=None), E_ARG), (dict(clen=at(46) + 2), E_ARG), (dict(out=at(47) + 1), E_ARG),
    (dict(v=heads(12, 4)), E_ARG), (dict(c=cache(head_dim=32)), E_UNS), (dict(c=cache(page_size=12)), E_UNS)])
def test_append_rejects(kw, code):
    assert append(**kw) == code


def inside(i, first, h, S=3, total=8, **kw):
    """Heads first .. first + h of a tensor of `total` heads at place i."""
    return heads(i, h, data=at(i) + first * 64 * 2, ss=total * 64, sb=S * total * 64, **kw)


@pytest.mark.parametrize("kw", [
    dict(q_out=heads(9)), dict(q_out=heads(8, data=at(8) + 128)), dict(k_out=heads(10, 2)), dict(q_out=heads(45)),
    dict(q_out=heads(40)), dict(k_out=heads(41, 2)), dict(k_out=heads(42, 2)), dict(q_out=heads(43)),
    dict(k_out=heads(44, 2)), dict(k_out=heads(8, 2)),
    dict(q_out=inside(8, 0, 4)),                                   # over its dense input, not in place
    dict(q=inside(8, 0, 4), k=inside(8, 4, 2), q_out=inside(8, 1, 4)),
    dict(q=inside(8, 0, 4), k=inside(8, 4, 2), q_out=inside(8, 0, 4), k_out=inside(8, 5, 2)),
    dict(q=inside(8, 0, 4), k=inside(8, 4, 2), q_out=inside(8, 4, 4)),
    dict(q_out=inside(8, 6, 4, total=10), k_out=inside(8, 8, 2, total=10))])
def test_forward_rejects_overlaps(kw):
    assert fwd(**kw) == E_ALIAS


@pytest.mark.parametrize("kw", [
    dict(dq=heads(8)), dict(dk=heads(9, 2)), dict(dq=heads(9)), dict(dk=heads(10, 2)), dict(dgq=at(47)), dict(dgk=at(48)),
    dict(dgq=at(10) + 64), dict(ws=at(8)), dict(ws=at(12)), dict(dgq=at(43)), dict(dq=heads(13)), dict(dk=heads(12, 2)),
    dict(ws=at(40)), dict(dq=heads(45)), dict(dq=heads(12, data=at(12) + 128)), dict(dgk=at(45))])
def test_backward_rejects_overlaps(kw):
    assert bwd(**kw) == E_ALIAS


@pytest.mark.parametrize("kw", [
    dict(q_out=heads(0)), dict(q_out=heads(9)), dict(q_out=heads(12)), dict(q_out=heads(46)), dict(q_out=heads(2)),
    dict(out=at(46)), dict(out=at(10)), dict(out=at(9)), dict(out=at(2)), dict(k=heads(0, 2)), dict(v=heads(1, 2)),
    dict(q=heads(1)), dict(rope=rope(pos=FAKE + 64)), dict(out=FAKE + 16), dict(row_len=at(47)), dict(row_len=at(10))])
def test_append_rejects_overlaps(kw):
    assert append(**kw) == E_ALIAS


@NO_GPU
def test_valid_calls_reach_the_device():
    assert fwd() == E_HIP and bwd() == E_HIP and append() == E_HIP
    assert fwd(norm=None, rope=None, row_len=None) == E_HIP and fwd(rope=rope(axis=None, axes=1)) == E_HIP
    assert fwd(q_out=heads(8)) == E_HIP and bwd(dq=heads(12), dk=heads(13, 2)) == E_HIP
    assert fwd(q=None, q_out=None) == E_HIP and fwd(k=None, k_out=None, D=128, q=heads(8, D=128), q_out=heads(10, D=128)) == E_HIP
    # one projection's output, in place, and both outputs in one tensor
    fused = dict(q=inside(8, 0, 4), k=inside(8, 4, 2))
    assert fwd(**fused) == E_HIP and fwd(q_out=inside(8, 0, 4), k_out=inside(8, 4, 2), **fused) == E_HIP
    assert fwd(q_out=inside(10, 0, 4), k_out=inside(10, 4, 2)) == E_HIP
    assert append(v=inside(8, 6, 2), q_out=inside(8, 0, 4), **fused) == E_HIP
    assert bwd(dgq=None, dgk=None, ws=None, ws_bytes=0, norm=None) == E_HIP and bwd(dgq=None) == E_HIP
    assert append(q=None, q_out=None, out=None) == E_HIP
    assert fwd(q_out=heads(10, ss=64, sh=192, sb=800)) == E_HIP  # heads outermost in a sequence


def test_sizes():
    size = skv.speechkv_norm_rope_bwd_workspace_bytes
    for B, S, Hq, Hkv in ((1, 1, 1, 0), (1, 1, 0, 3), (2, 3, 4, 2), (8, 1596, 16, 8), (65535, 200, 64, 8), (1, 2 ** 24 - 1, 1, 1)):
        for D in (64, 128):  # a sum a block, one block at least and about two thousand at most
            assert D * 4 <= size(B, S, Hq, Hkv, D) <= 2050 * D * 4
    for bad in ((0, 3, 4, 2, 64), (2, 0, 4, 2, 64), (2, 3, 0, 0, 64), (2, 3, -1, 2, 64), (2, 3, 4, 2, 32),
                (65535, 1 << 20, 4, 2, 64)):
        assert size(*bad) == 0


# ------------------------------------------------------------------ binding

def host():
    z = lambda *s: torch.zeros(*s, dtype=torch.bfloat16)  # noqa: E731
    i = lambda *s: torch.zeros(*s, dtype=torch.int32)  # noqa: E731
    return dict(q=z(2, 3, 4, 64), k=z(2, 3, 2, 64), q_out=z(2, 3, 4, 64), k_out=z(2, 3, 2, 64)), i


@pytest.mark.parametrize("kw", [
    dict(k=torch.zeros(2, 3, 2, 64)), dict(k=torch.zeros(2, 4, 2, 64, dtype=torch.bfloat16)),
    dict(q=torch.zeros(2, 3, 4, 128, dtype=torch.bfloat16)[..., ::2]), dict(q=None, k=None),
    dict(q_out=torch.zeros(2, 3, 4, 64)), dict(gamma_q=torch.ones(32)), dict(gamma_k=torch.ones(64).double()),
    dict(gamma_q=torch.ones(64), normalise=False), dict(row_len=torch.zeros(2)),
    dict(row_len=torch.zeros(3, dtype=torch.int32)), dict(q=torch.zeros(3, 4, 64, dtype=torch.bfloat16)),
    dict(rope=skv.Rope(torch.zeros(2, 4, dtype=torch.int32), torch.zeros(32)))])
def test_binding_refuses(kw):
    a, _ = host()
    a.update(kw)
    with pytest.raises(ValueError):
        skv.speechkv_norm_rope(**a, stream=0)


def test_binding_refuses_rotations_and_other_descriptions():
    a, i = host()
    for args in ((torch.zeros(2, 3), torch.zeros(8)), (i(3), torch.zeros(8)), (i(2, 3), torch.zeros(8).double()),
                 (i(2, 3), torch.zeros(8), i(7)), (i(2, 3), torch.zeros(8), None, 3), (i(2, 6)[:, ::2], torch.zeros(8))):
        with pytest.raises(ValueError):
            skv.Rope(*args)
    with pytest.raises(TypeError):
        skv.speechkv_norm_rope(**a, rope=i(2, 3), stream=0)
    with pytest.raises(skv.SpeechKVError):  # more elements than a head has
        skv.speechkv_norm_rope(**a, rope=skv.Rope(i(2, 3), torch.zeros(40)), stream=0)
    with pytest.raises(ValueError):  # another batch's cache
        c = skv.PagedKV(torch.zeros(8, 2, 16, 64, dtype=torch.bfloat16), torch.zeros(8, 2, 16, 64, dtype=torch.bfloat16),
                        i(3, 4))
        skv.speechkv_norm_append_kv(a["q"], a["k"], a["k"].clone(), c, i(2), a["q_out"], stream=0)
    with pytest.raises(ValueError):
        skv.speechkv_norm_rope_bwd(a["q"], a["k"], a["q_out"], a["k_out"], a["q"].clone(), a["k"].clone(),
                                   dgamma_q=torch.zeros(64, dtype=torch.bfloat16), stream=0)


def test_packed_descriptions_fill_their_structures():
    a, i = host()
    q = a["q"][:, :, 1:3]
    h = skv._Heads.from_buffer_copy(skv._heads(q, 2, 3, 64, torch.bfloat16, -1))
    assert (h.data, h.stride_b, h.stride_s, h.stride_h, h.num_heads) == (q.data_ptr(), 768, 256, 64, 2)
    r = skv.Rope(i(3, 2, 3), torch.zeros(8), i(8), skv.ROPE_PAIRS)
    s = skv._Rope.from_buffer_copy(r._packed)
    assert (s.num_axes, s.rot_dim, s.layout) == (3, 16, 1) and s.axis and s.positions and s.inv_freq


# ------------------------------------------------- the gradients' oracle

@pytest.mark.parametrize("pairs", [False, True])
@pytest.mark.parametrize("eps", [1e-2, None])
def test_reference_gradients_by_differences(pairs, eps):
    rng = np.random.default_rng(5)
    S, H, D = 2, 2, 16
    x, dy, gamma = rng.normal(size=(S, H, D)), rng.normal(size=(S, H, D)), rng.normal(size=D)
    rot = (rng.integers(0, 50, (2, S)), rng.random(4), np.array([0, 1, 1, 0]), pairs)
    loss = lambda x, g: float((norm_ref.forward(x, g, eps, rot, 0.0)[0] * dy).sum())  # noqa: E731
    dx, _, dg, _ = norm_ref.backward(x, dy, gamma, eps, rot, 0.0)
    step = 1e-5
    for at_ in np.ndindex(x.shape):
        e = np.zeros_like(x)
        e[at_] = step
        assert abs((loss(x + e, gamma) - loss(x - e, gamma)) / (2 * step) - dx[at_]) < 1e-8
    if eps is not None:
        for j in range(D):
            e = np.zeros(D)
            e[j] = step
            assert abs((loss(x, gamma + e) - loss(x, gamma - e)) / (2 * step) - dg[j]) < 1e-8


def test_reference_rotation_is_a_complex_product():
    rng = np.random.default_rng(6)
    x, pos = rng.normal(size=(3, 2, 8)), rng.integers(-9, 9, (1, 3))
    inv = rng.random(4)
    y = norm_ref.turned(x, pos, inv, np.zeros(4, dtype=int), True)[0]
    z = (x[..., 0::2] + 1j * x[..., 1::2]) * np.exp(1j * pos[0][:, None, None] * inv)
    assert np.allclose(y[..., 0::2], z.real) and np.allclose(y[..., 1::2], z.imag)
    y = norm_ref.turned(x, pos, inv, np.zeros(4, dtype=int), False)[0]
    z = (x[..., :4] + 1j * x[..., 4:]) * np.exp(1j * pos[0][:, None, None] * inv)
    assert np.allclose(y[..., :4], z.real) and np.allclose(y[..., 4:], z.imag)
