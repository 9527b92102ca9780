"""The calls of include/speechkv_shared.h on the CPU: the header and the library
agree, invalid arguments are rejected before any HIP call, and the binding
refuses what it cannot pass on (no kernel is launched)."""
import ctypes
import os
import re
import shutil
import subprocess

import numpy as np
import pytest
import torch

import shared_ref
from paper_2607_06827_amd import speechkv as skv
from test_abi import FAKE, NO_GPU, cache
from test_draft_abi import E_ALIAS, E_ARG, E_HIP, E_UNS, E_WS, at
from test_norm_abi import heads

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HEADER = os.path.join(ROOT, "include", "speechkv_shared.h")
lib = skv._lib
INF, NAN = float("inf"), float("nan")


def test_every_declared_symbol_is_exported():
    text = re.sub(r"/\*.*?\*/", "", open(HEADER).read(), flags=re.S)
    names = set(re.findall(r"\b(speechkv_[a-z0-9_]+)\s*\(", text))
    assert names == {"speechkv_shared_attn", "speechkv_shared_num_splits", "speechkv_shared_workspace_bytes",
                     "speechkv_attn_weights", "speechkv_evict"}
    for n in names:
        assert hasattr(lib, n) and callable(getattr(skv, n)), n
    defs = dict(re.findall(r"#define SPEECHKV_(\w+) (\d+)", open(HEADER).read()))
    assert {n: int(v) for n, v in defs.items()} == {"MAX_EVICT_LAYERS": skv.MAX_EVICT_LAYERS}


@pytest.mark.skipif(shutil.which("gcc") is None, reason="needs gcc")
def test_header_compiles_as_c_and_cxx(tmp_path):
    for std, cc, name in (("c11", "gcc", "x.c"), ("c++17", "g++", "x.cc")):
        src = tmp_path / name
        src.write_text('#include "speechkv_shared.h"\n#include <stdio.h>\n'
                       'int main(void) { printf("%zu", sizeof(speechkv_evict_layer)); return 0; }\n')
        exe = tmp_path / (name + ".exe")
        subprocess.run([cc, f"-std={std}", "-Wall", "-Wextra", "-Werror", "-pedantic",
                        f"-I{os.path.join(ROOT, 'include')}", str(src), "-o", str(exe)], check=True)
        size = subprocess.run([str(exe)], check=True, capture_output=True, text=True).stdout
        assert int(size) == ctypes.sizeof(skv._EvictLayer)


# ------------------------------------------------------------ shared prefixes

def shared(p=None, c=None, **kw):
    a = dict(q=at(8), batch=5, hq=4, plen=at(9), max_prefix=100, start=at(10), groups=2, most=3, clen=at(11),
             max_len=100, scale=0.125, splits=0, out=at(12), lse=at(13), ws=at(64), ws_bytes=1 << 30)
    a.update(kw)
    p = p or cache(k_pages=at(4), v_pages=at(5), block_table=at(6))
    c = c or cache()
    return lib.speechkv_shared_attn(a["q"], a["batch"], a["hq"], ctypes.byref(p), a["plen"], a["max_prefix"], a["start"],
                                    a["groups"], a["most"], ctypes.byref(c), a["clen"], a["max_len"], a["scale"],
                                    a["splits"], a["out"], a["lse"], a["ws"], a["ws_bytes"], None)


@pytest.mark.parametrize("kw,code", [
    (dict(q=None), E_ARG), (dict(out=None), E_ARG), (dict(plen=None), E_ARG), (dict(start=None), E_ARG),
    (dict(clen=None), E_ARG), (dict(batch=0), E_ARG), (dict(batch=65536), E_ARG), (dict(groups=0), E_ARG),
    (dict(groups=65536), E_ARG), (dict(most=0), E_ARG), (dict(most=6), E_ARG), (dict(max_prefix=-1), E_ARG),
    (dict(max_prefix=129), E_ARG), (dict(max_len=-1), E_ARG), (dict(max_len=129), E_ARG), (dict(splits=-1), E_ARG),
    (dict(splits=1025), E_ARG), (dict(scale=0.0), E_ARG), (dict(scale=NAN), E_ARG), (dict(scale=INF), E_ARG),
    (dict(hq=0), E_ARG), (dict(hq=5), E_ARG), (dict(hq=6), E_UNS), (dict(q=at(8) + 8), E_ARG),
    (dict(out=at(12) + 2), E_ARG), (dict(lse=at(13) + 2), E_ARG), (dict(plen=at(9) + 1), E_ARG),
    (dict(start=at(10) + 2), E_ARG), (dict(clen=at(11) + 2), E_ARG), (dict(ws=None), E_WS), (dict(ws=at(64) + 4), E_WS),
    (dict(ws_bytes=100), E_WS), (dict(p=cache(head_dim=128)), E_ARG), (dict(p=cache(num_kv_heads=4)), E_ARG),
    (dict(p=cache(dtype=skv.DTYPE_F32)), E_ARG), (dict(p=cache(head_dim=32)), E_UNS), (dict(c=cache(page_size=12)), E_UNS)])
def test_shared_rejects(kw, code):
    assert shared(**kw) == code


@pytest.mark.parametrize("kw", [
    dict(out=at(8)), dict(out=at(9)), dict(out=at(10)), dict(out=at(11)), dict(out=at(4)), dict(out=FAKE), dict(out=at(6)),
    dict(out=at(2)), dict(lse=at(12)), dict(lse=at(8)), dict(lse=at(5) + 64), dict(lse=at(10)), dict(ws=at(12)),
    dict(ws=at(13) - 16), dict(ws=at(8)), dict(ws=at(1)), dict(ws=at(9))])
def test_shared_rejects_overlaps(kw):
    assert shared(**kw) == E_ALIAS


def test_shared_refuses_what_a_launch_cannot_count():
    wide = dict(batch=65535, groups=65535, most=65535, hq=16, p=cache(k_pages=at(4), v_pages=at(5), block_table=1 << 60,
                                                                     num_kv_heads=2),
                q=1 << 50, out=1 << 51, lse=1 << 52, ws=1 << 53, ws_bytes=1 << 50, plen=1 << 54, start=1 << 55, clen=1 << 56)
    assert shared(**wide) == E_UNS
    far = cache(page_size=256, max_pages_per_seq=8388607)
    assert shared(c=far, max_len=2 ** 31 - 8191, out=1 << 52, lse=1 << 53) == E_UNS


def test_shared_sizes():
    split, ws = skv.speechkv_shared_num_splits, skv.speechkv_shared_workspace_bytes
    BF, F32 = torch.bfloat16, torch.float32
    good = (5, 2, 3, 4, 2, 64, 100, 100)
    for i, bad in ((0, 0), (1, 0), (2, 0), (2, 6), (3, 3), (4, 0), (5, 32), (6, -1), (7, -1)):
        args = list(good)
        args[i] = bad
        assert split(*args[:6], BF, *args[6:]) == -1 and ws(*args) == 0
    assert split(*good[:6], torch.float16, *good[6:]) == -1
    assert ws(*good, -1) == 0 and ws(*good, 1025) == 0
    for B, n, most in ((1, 1, 1), (8, 1, 8), (64, 1, 64), (40, 6, 11), (65535, 3, 60000)):
        for D in (64, 128):
            for P in (0, 1, 126, 1500, 7532, 65536):
                for L in (0, 1, 40, 3000):
                    counts = [split(B, n, most, 16, 8, D, dt, P, L) for dt in (BF, F32)]
                    assert all(1 <= s <= 64 for s in counts)
                    assert ws(B, n, most, 16, 8, D, P, L) >= B * 16 * (max(counts) + 1) * (D + 2) * 4
                    assert ws(B, n, most, 16, 8, D, P, L, 9) >= B * 16 * 10 * (D + 2) * 4


@NO_GPU
def test_shared_valid_calls_reach_the_device():
    assert shared() == E_HIP and shared(lse=None) == E_HIP and shared(max_prefix=0, max_len=0) == E_HIP
    assert shared(p=cache(block_table=at(6), page_size=64, max_pages_per_seq=2)) == E_HIP  # one pool, other pages
    need = skv.speechkv_shared_workspace_bytes(5, 2, 3, 4, 2, 64, 100, 100, 7)
    assert shared(splits=7, ws_bytes=need) == E_HIP and shared(splits=7, ws_bytes=need - 4) == E_WS


# -------------------------------------------------------------- entry weights

def weights(c=None, **kw):
    a = dict(q=heads(8), batch=2, rows=3, lse=at(9), lb=12, lh=3, ls=1, visible=at(10), clen=at(11), max_len=100,
             scale=0.125, w=at(12), out=at(13), capacity=120)
    a.update(kw)
    c = c or cache()
    q = None if a["q"] is None else ctypes.byref(a["q"])
    return lib.speechkv_attn_weights(q, a["batch"], a["rows"], a["lse"], a["lb"], a["lh"], a["ls"], a["visible"],
                                     ctypes.byref(c), a["clen"], a["max_len"], a["scale"], a["w"], a["out"],
                                     a["capacity"], None)


@pytest.mark.parametrize("kw,code", [
    (dict(q=None), E_ARG), (dict(lse=None), E_ARG), (dict(clen=None), E_ARG), (dict(out=None), E_ARG),
    (dict(batch=0), E_ARG), (dict(batch=65536), E_ARG), (dict(rows=0), E_ARG), (dict(rows=1 << 24), E_ARG),
    (dict(capacity=0), E_ARG), (dict(capacity=99), E_ARG), (dict(max_len=-1), E_ARG), (dict(max_len=129, capacity=200), E_ARG),
    (dict(scale=0.0), E_ARG), (dict(scale=NAN), E_ARG), (dict(scale=INF), E_ARG), (dict(lb=-1), E_ARG), (dict(lh=-1), E_ARG),
    (dict(ls=-1), E_ARG), (dict(lb=1 << 62), E_ARG), (dict(lse=at(9) + 2), E_ARG), (dict(visible=at(10) + 1), E_ARG),
    (dict(clen=at(11) + 2), E_ARG), (dict(w=at(12) + 2), E_ARG), (dict(out=at(13) + 1), E_ARG),
    (dict(q=heads(8, h=5)), E_ARG), (dict(q=heads(8, h=6)), E_UNS), (dict(q=heads(8, sb=4)), E_ARG),
    (dict(q=heads(8, data=at(8) + 8)), E_ARG), (dict(c=cache(head_dim=32)), E_UNS),
    (dict(c=cache(page_size=256, max_pages_per_seq=8388607), max_len=2 ** 31 - 8191, capacity=2 ** 31 - 1), E_UNS),
    (dict(c=cache(page_size=256, max_pages_per_seq=8388607, num_kv_heads=60000), q=heads(8, h=60000), max_len=10 ** 6,
          capacity=10 ** 6), E_UNS),
    (dict(c=cache(num_kv_heads=60000, num_pages=1), q=heads(8, h=60000, sb=0, ss=0), batch=65535, rows=1, lb=0, lh=0,
          capacity=2 ** 31 - 1, max_len=1), E_UNS),  # (blocks before bytes)
    (dict(c=cache(num_kv_heads=60000, num_pages=1), q=heads(8, h=60000, sb=0, ss=0), batch=65535, rows=1, lb=0, lh=0,
          capacity=2 ** 31 - 1, max_len=0), E_ARG)])
def test_weights_rejects(kw, code):
    assert weights(**kw) == code


@pytest.mark.parametrize("kw", [dict(out=at(8)), dict(out=at(9)), dict(out=at(10)), dict(out=at(11)), dict(out=FAKE),
                                dict(out=at(2)), dict(out=at(12) + 4)])
def test_weights_rejects_overlaps(kw):
    assert weights(**kw) == E_ALIAS


@NO_GPU
def test_weights_refuse_launches_of_two_to_the_32_threads():
    # 65535 sequences of 128 heads: a block of 512 threads for every 128 keys at most with
    # many rows, of 256 threads for more keys with few
    big = dict(c=cache(num_kv_heads=128, num_pages=1, max_pages_per_seq=20), q=heads(8, h=128, sb=0, ss=0, sh=64), batch=65535,
               lse=at(9), lb=0, lh=0, ls=0, visible=None, capacity=200, w=None, out=at(10 ** 6))
    assert weights(**{**big, "rows": 64, "max_len": 129}) == E_UNS
    assert weights(**{**big, "rows": 64, "max_len": 64}) == E_HIP
    assert weights(**{**big, "rows": 1, "max_len": 129}) == E_HIP


@NO_GPU
def test_weights_valid_calls_reach_the_device():
    assert weights() == E_HIP and weights(visible=None, w=None) == E_HIP and weights(w=at(13)) == E_HIP
    assert weights(lb=0, lh=1, ls=4) == E_HIP and weights(out=at(1)) == E_HIP  # (values are not read)
    assert weights(max_len=0) == skv.OK  # nothing to do


# ------------------------------------------------------------------ eviction

def layer(i=0, clen=None, out=None, w=None, w_out=None, kept=None, **kw):
    base = 16 + 10 * i
    c = cache(k_pages=at(base), v_pages=at(base + 1), block_table=at(base + 2), **kw)
    return skv._EvictLayer(c, at(base + 3) if clen is None else clen, out, at(base + 4) if w is None else w,
                           at(base + 5) if w_out is None else w_out, at(base + 6) if kept is None else kept)


def evict(layers=None, **kw):
    a = dict(batch=2, keep=at(8), max_keep=50, capacity=100, first=4, recent=8)
    a.update(kw)
    layers = [layer()] if layers is None else layers
    arr = (skv._EvictLayer * max(1, len(layers)))(*layers)
    return lib.speechkv_evict(ctypes.byref(arr), a.get("count", len(layers)), a["batch"], a["keep"], a["max_keep"],
                              a["capacity"], a["first"], a["recent"], None)


@pytest.mark.parametrize("kw,code", [
    (dict(keep=None), E_ARG), (dict(keep=at(8) + 2), E_ARG), (dict(batch=0), E_ARG), (dict(batch=65536), E_ARG),
    (dict(max_keep=0), E_ARG), (dict(capacity=0), E_ARG), (dict(first=-1), E_ARG), (dict(recent=-1), E_ARG),
    (dict(count=0), E_ARG), (dict(count=257), E_ARG), (dict(count=-1), E_ARG),
    (dict(layers=[layer(num_kv_heads=60000)], batch=65535, capacity=2 ** 31 - 1), E_ARG),   # rows past 2^62 bytes
    (dict(layers=[layer(num_kv_heads=60000)], batch=65535, max_keep=2 ** 31 - 1), E_ARG)])
def test_evict_rejects(kw, code):
    assert evict(**kw) == code
    assert lib.speechkv_evict(None, 1, 1, at(8), 1, 1, 0, 0, None) == E_ARG


@pytest.mark.parametrize("layers,code", [
    ([layer(clen=0)], E_ARG), ([layer(w=0)], E_ARG), ([layer(w_out=0)], E_ARG), ([layer(kept=0)], E_ARG),
    ([layer(clen=at(19) + 2)], E_ARG), ([layer(out=at(23) + 1)], E_ARG), ([layer(w=at(20) + 2)], E_ARG),
    ([layer(w_out=at(21) + 2)], E_ARG), ([layer(kept=at(22) + 1)], E_ARG), ([layer(head_dim=32)], E_UNS),
    ([layer(page_size=12)], E_UNS), ([layer(), layer(1, head_dim=128)], E_ARG), ([layer(), layer(1, num_kv_heads=4)], E_ARG),
    ([layer(), layer(1, dtype=skv.DTYPE_F32)], E_ARG),
    ([layer(out=at(19))], E_ALIAS), ([layer(out=at(8))], E_ALIAS), ([layer(out=at(16) + 4)], E_ALIAS),
    ([layer(out=at(20))], E_ALIAS), ([layer(out=at(21))], E_ALIAS), ([layer(out=at(22))], E_ALIAS),
    ([layer(w_out=at(16))], E_ALIAS), ([layer(w_out=at(17))], E_ALIAS), ([layer(w_out=at(18))], E_ALIAS),
    ([layer(w_out=at(20) + 4)], E_ALIAS), ([layer(w_out=at(22))], E_ALIAS), ([layer(w_out=at(8))], E_ALIAS),
    ([layer(kept=at(8))], E_ALIAS), ([layer(kept=at(20))], E_ALIAS), ([layer(kept=at(17))], E_ALIAS),
    ([layer(kept=at(19))], E_ALIAS), ([layer(kept=at(18))], E_ALIAS), ([layer(w=at(16))], E_ALIAS),
    ([layer(), layer(1, w_out=at(21))], E_ALIAS), ([layer(), layer(1, w_out=at(20))], E_ALIAS),
    ([layer(), layer(1, kept=at(22) + 4)], E_ALIAS), ([layer(out=at(60)), layer(1, out=at(60) + 4)], E_ALIAS),
    ([layer(), layer(1, clen=at(16) + 4)], E_ALIAS), ([layer(w_out=at(29)), layer(1)], E_ALIAS),
    ([layer(w=at(21)), layer(1, w=at(21))], E_ALIAS)])  # one layer's in place, and the other's input
def test_evict_rejects_layers(layers, code):
    assert evict(layers) == code


def test_evict_refuses_lengths_past_31_bits_with_a_stretch():
    assert evict([layer(num_kv_heads=1)], batch=1, capacity=2 ** 31 - 8191) == E_UNS
    assert evict([layer(num_kv_heads=1)], batch=1, capacity=2 ** 31 - 1) == E_UNS


@NO_GPU
def test_evict_valid_calls_reach_the_device():
    assert evict() == E_HIP and evict([layer(out=at(23)), layer(1, page_size=64, max_pages_per_seq=3)]) == E_HIP
    assert evict([layer(w=at(21))]) == E_HIP  # in place
    both = layer(1)
    both.cache.k_pages, both.cache.v_pages, both.weights = at(16), at(17), at(20)
    assert evict([layer(), both]) == E_HIP  # layers of one pool, and of one set of weights
    assert evict(first=2 ** 31 - 1, recent=2 ** 31 - 1) == E_HIP


# ------------------------------------------------------------------ binding

def host():
    z = lambda *s: torch.zeros(*s, dtype=torch.bfloat16)  # noqa: E731
    i = lambda *s: torch.zeros(*s, dtype=torch.int32)  # noqa: E731
    c = skv.PagedKV(z(8, 2, 16, 64), z(8, 2, 16, 64), i(3, 4))
    p = skv.PagedKV(z(8, 2, 16, 64), z(8, 2, 16, 64), i(2, 4))
    return dict(q=z(3, 4, 64), prefix=p, prefix_len=i(2), max_prefix_len=5, group_start=i(3), max_group=2, cache=c,
                cache_len=i(3), max_cache_len=5, out=z(3, 4, 64), stream=0), i, z


@pytest.mark.parametrize("kw", [
    dict(out=torch.zeros(3, 4, 64)), dict(q=torch.zeros(2, 4, 64, dtype=torch.bfloat16)), dict(lse=torch.zeros(4, 3).t()),
    dict(lse=torch.zeros(3, 4, dtype=torch.bfloat16)), dict(prefix_len=torch.zeros(3, dtype=torch.int32)),
    dict(group_start=torch.zeros(2, dtype=torch.int32)), dict(cache_len=torch.zeros(3)),
    dict(workspace=torch.zeros(64, 64).t())])
def test_binding_refuses_shared(kw):
    a, _, _ = host()
    a.update(kw)
    with pytest.raises(ValueError):
        skv.speechkv_shared_attn(**a)


def test_binding_refuses_counts_and_descriptions():
    a, i, z = host()
    spans = skv.Spans(i(3), i(3), i(3), 0, 8)
    for kw in (dict(prefix=spans), dict(cache=spans)):
        with pytest.raises(TypeError):
            skv.speechkv_shared_attn(**dict(a, **kw))
    for kw in (dict(max_group=2 ** 32 + 2), dict(max_prefix_len=2 ** 32 + 5), dict(max_cache_len=-1),
               dict(num_splits=2 ** 32 + 1)):
        with pytest.raises(skv.SpeechKVError) as e:
            skv.speechkv_shared_attn(**dict(a, workspace=z(1 << 16), **kw))
        assert e.value.status == E_ARG
    with pytest.raises(ValueError):  # other heads
        skv.speechkv_shared_attn(**dict(a, prefix=skv.PagedKV(z(8, 4, 16, 64), z(8, 4, 16, 64), i(2, 4))))


@pytest.mark.parametrize("kw", [
    dict(lse=torch.zeros(3, 2, 4)), dict(lse=torch.zeros(3, 4, 2, dtype=torch.bfloat16)),
    dict(weights_out=torch.zeros(3, 4, 9)), dict(weights=torch.zeros(3, 2, 8)), dict(weights=torch.zeros(3, 2, 9).double()),
    dict(weights_out=torch.zeros(3, 9, 2).transpose(1, 2)), dict(visible=torch.zeros(3, 2)),
    dict(visible=torch.zeros(3, 1, dtype=torch.int32)), dict(q=torch.zeros(2, 2, 4, 64, dtype=torch.bfloat16)),
    dict(q=torch.zeros(3, 4, 64, dtype=torch.bfloat16)), dict(cache_len=torch.zeros(2, dtype=torch.int32))])
def test_binding_refuses_weights(kw):
    a, i, z = host()
    x = dict(q=z(3, 2, 4, 64), lse=torch.zeros(3, 4, 2), cache=a["cache"], cache_len=i(3), max_cache_len=5,
             weights_out=torch.zeros(3, 2, 9), stream=0)
    x.update(kw)
    with pytest.raises(ValueError):
        skv.speechkv_attn_weights(**x)


def test_binding_refuses_evict():
    a, i, z = host()
    c, f = a["cache"], lambda *s: torch.zeros(*s)  # noqa: E731
    good = ([c], [i(3)], [i(3)], [f(3, 2, 9)], [f(3, 2, 9)], [i(3, 2, 5)])
    for at_, bad in ((1, []), (1, [i(2)]), (1, [f(3)]), (2, [i(3), None]), (3, [f(3, 2, 8)]), (4, [f(3, 1, 9)]),
                     (4, [f(3, 2, 9).double()]), (5, [f(3, 2, 5)]), (5, [i(3, 3, 5)]), (5, [i(3, 5, 2).transpose(1, 2)])):
        args = list(good)
        args[at_] = bad
        with pytest.raises(ValueError):
            skv.EvictStack(*args)
    stack = skv.EvictStack(*good)
    layer_, = (skv._EvictLayer * 1).from_buffer_copy(stack._packed)
    assert layer_.weights == good[3][0].data_ptr() and layer_.kept == good[5][0].data_ptr()
    assert (stack.batch, stack.capacity, stack.max_keep, stack.num_layers) == (3, 9, 5, 1)
    with pytest.raises(TypeError):
        skv.speechkv_evict(c, i(3), 0, 0, stream=0)
    with pytest.raises(ValueError):
        skv.speechkv_evict(stack, i(2), 0, 0, stream=0)
    for n in (2 ** 32, -1):
        with pytest.raises(skv.SpeechKVError):
            skv.speechkv_evict(stack, i(3), n, 0, stream=0)
    with pytest.raises(skv.SpeechKVError):
        skv.speechkv_evict(skv.EvictStack([], [], None, [], [], []), i(0), 0, 0, stream=0)


# -------------------------------------------------------------- the references

@pytest.mark.parametrize("mode", [0, 1])
def test_visible_slots_by_the_rule(mode):
    """A key is visible from its own row (text), its window's last or first frame."""
    for segs in ([(2, 5), (1, 0)], [(0, 3)], [(0, 0), (4, 8), (2, 1), (0, 7)], [(3, 0)], [(0, 4), (0, 4)]):
        for w in (1, 2, 4, 9):
            starts, rows = [], 0
            for text, speech in segs:
                starts += [rows + i for i in range(text)]
                rows += text
                for f in range(0, speech, w):
                    starts.append(rows + (f if mode else min(f + w, speech) - 1))
                rows += speech
            want = [sum(s <= p for s in starts) for p in range(rows)]
            assert skv.visible_slots([segs], w, 3, 3, mode, device="cpu").tolist() == [want]
            if w > 1:
                assert skv.visible_slots([segs], w, 2, 3, mode, device="cpu").tolist() == [list(range(1, rows + 1))]


def test_reference_eviction():
    nan = float("nan")
    w = np.array([0.0, 5.0, nan, -0.0, 2.0, 2.0, -INF, 9.0])
    assert shared_ref.kept_slots(w, 3, 0, 0) == [1, 4, 7]
    assert shared_ref.kept_slots(w, 5, 0, 0) == [0, 1, 4, 5, 7]
    assert shared_ref.kept_slots(w, 6, 0, 0) == [0, 1, 3, 4, 5, 7]
    assert shared_ref.kept_slots(w, 7, 0, 0) == [0, 1, 3, 4, 5, 6, 7]
    assert shared_ref.kept_slots(w, 3, 1, 2) == [0, 6, 7] and shared_ref.kept_slots(w, 4, 1, 2) == [0, 1, 6, 7]
    assert shared_ref.kept_slots(w, 2, 5, 5) == [0, 1] and shared_ref.kept_slots(w, 0, 5, 5) == []
    assert shared_ref.kept_slots(w, 9, 1, 1) == list(range(8))


def test_reference_weights_are_the_softmax():
    rng = np.random.default_rng(0)
    q, K = rng.normal(size=(3, 8)), rng.normal(size=(5, 8))
    z = q @ K.T * 0.3
    seen = np.array([5, 2, 0])
    lse = np.array([np.log(np.exp(z[i, :s]).sum()) if s else -np.inf for i, s in enumerate(seen)])
    got, _ = shared_ref.gathered(q, lse, seen, K, 0.3, np.zeros(5))
    want = np.exp(z[0]) / np.exp(z[0]).sum()
    want[:2] += np.exp(z[1, :2]) / np.exp(z[1, :2]).sum()
    assert np.allclose(got, want)
