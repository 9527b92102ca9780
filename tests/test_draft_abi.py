"""The calls of include/speechkv_draft.h on the CPU: the header and the library
agree, invalid arguments are rejected before any HIP call, and the binding
refuses what it cannot pass on (no kernel is launched)."""
import ctypes
import os
import re
import shutil
import subprocess

import pytest
import torch

from paper_2607_06827_amd import speechkv as skv
from test_abi import FAKE, cache

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HEADER = os.path.join(ROOT, "include", "speechkv_draft.h")
lib = skv._lib
E_ARG, E_UNS, E_WS, E_ALIAS, E_HIP = (skv.ERR_INVALID_ARG, skv.ERR_UNSUPPORTED, skv.ERR_WORKSPACE,
                                      skv.ERR_ALIAS, skv.ERR_HIP)


def at(i):
    return FAKE + (i << 24)


def test_every_declared_symbol_is_exported():
    text = re.sub(r"/\*.*?\*/", "", open(HEADER).read(), flags=re.S)
    names = set(re.findall(r"\b(speechkv_[a-z0-9_]+)\s*\(", text))
    assert names == {"speechkv_append_kv", "speechkv_tree_attn", "speechkv_tree_num_splits",
                     "speechkv_tree_workspace_bytes", "speechkv_tree_commit"}
    for n in names:
        assert hasattr(lib, n) and callable(getattr(skv, n)), n


def test_binding_constants_match_header():
    defs = dict(re.findall(r"#define SPEECHKV_(\w+) (\d+)", open(HEADER).read()))
    assert set(defs) == {"MAX_TREE_NODES", "MAX_COMMIT_LAYERS", "ROPE_HALVES", "ROPE_PAIRS"}
    for name, value in defs.items():
        assert int(value) == getattr(skv, name), name


@pytest.mark.skipif(shutil.which("gcc") is None, reason="needs gcc")
def test_header_compiles_as_c_and_cxx(tmp_path):
    for std, cc, name in (("c11", "gcc", "x.c"), ("c++17", "g++", "x.cc")):
        src = tmp_path / name
        src.write_text('#include "speechkv_draft.h"\n#include <stdio.h>\n'
                       'int main(void) { speechkv_layer_cache y; printf("%zu", sizeof y); return 0; }\n')
        exe = tmp_path / (name + ".exe")
        subprocess.run([cc, f"-std={std}", "-Wall", "-Wextra", "-Werror", "-pedantic",
                        f"-I{os.path.join(ROOT, 'include')}", str(src), "-o", str(exe)], check=True)
        size = subprocess.run([str(exe)], check=True, capture_output=True, text=True).stdout
        assert int(size) == ctypes.sizeof(skv._LayerCache)


# ------------------------------------------------------------------- append

def append(c=None, **kw):
    a = dict(q=at(8), qsb=3 * 4 * 64, qss=4 * 64, qsh=64, hq=4, k=at(9), v=at(10), sb=3 * 2 * 64, ss=2 * 64,
             sh=64, batch=2, n=3, new=None, pos=at(11), inv=at(12), rot=64, rope=0, clen=at(13), q_out=at(14),
             clen_out=None)
    a.update(kw)
    c = c or cache()
    return lib.speechkv_append_kv(a["q"], a["qsb"], a["qss"], a["qsh"], a["hq"], a["k"], a["v"], a["sb"], a["ss"],
                                  a["sh"], a["batch"], a["n"], a["new"], a["pos"], a["inv"], a["rot"], a["rope"],
                                  a["clen"], ctypes.byref(c), a["q_out"], a["clen_out"], None)


@pytest.mark.parametrize("kw,code", [
    (dict(k=None), E_ARG), (dict(v=None), E_ARG), (dict(clen=None), E_ARG), (dict(q=None), E_ARG),
    (dict(q_out=None), E_ARG), (dict(batch=0), E_ARG), (dict(batch=65536), E_ARG), (dict(n=0), E_ARG),
    (dict(n=1 << 24), E_ARG), (dict(rot=-16), E_ARG), (dict(rot=80), E_ARG), (dict(rot=24), E_ARG), (dict(rope=2), E_ARG),
    (dict(rope=-1), E_ARG), (dict(pos=None), E_ARG), (dict(inv=None), E_ARG), (dict(hq=3), E_ARG),
    (dict(hq=0), E_ARG), (dict(hq=6), E_UNS), (dict(sb=4), E_ARG), (dict(ss=-8), E_ARG), (dict(qsh=12), E_ARG),
    (dict(k=at(9) + 8), E_ARG), (dict(q=at(8) + 4), E_ARG), (dict(q_out=at(14) + 8), E_ARG),
    (dict(pos=at(11) + 2), E_ARG), (dict(clen=at(13) + 1), E_ARG), (dict(sb=1 << 61), E_ARG),
    (dict(qss=(1 << 62) - 8), E_ARG)])
def test_append_rejects(kw, code):
    assert append(**kw) == code


@pytest.mark.parametrize("kw", [
    dict(q_out=at(9)), dict(q_out=at(13)), dict(q_out=FAKE), dict(clen_out=at(13)), dict(clen_out=at(14)),
    dict(k=FAKE), dict(v=FAKE + (1 << 24)), dict(pos=FAKE + 64), dict(inv=FAKE + 64), dict(clen_out=at(2)),
    dict(new=at(14)), dict(clen_out=FAKE + 4),
    dict(q=at(14) + 16),                       # shifted in place
    dict(q=at(14), qss=8 * 64, qsb=24 * 64),   # in place, but not dense
])
def test_append_rejects_overlaps(kw):
    assert append(**kw) == E_ALIAS


def test_append_takes_queries_in_place_and_none_at_all():
    assert append(q=at(14)) == E_HIP
    assert append(q=at(14), n=1, qss=0, qsb=4 * 64) == E_HIP
    assert append(q=None, q_out=None, hq=0) == E_HIP
    assert append(rot=0, pos=None, inv=None) == E_HIP
    assert append(q=at(8), k=at(8) + 512, v=at(8) + 768, qss=512, qsb=1536, ss=512, sb=1536) == E_HIP  # one projection


# --------------------------------------------------------------------- tree

def tree(c=None, **kw):
    a = dict(q=at(8), batch=2, n=5, hq=4, clen=at(9), max_len=100, of=None, mask=at(10), ms=5, scale=0.125,
             splits=1, out=at(11), ws=None, ws_bytes=0)
    a.update(kw)
    c = c or cache()
    return lib.speechkv_tree_attn(a["q"], a["batch"], a["n"], a["hq"], ctypes.byref(c), a["clen"], a["max_len"],
                                  a["of"], a["mask"], a["ms"], a["scale"], a["splits"], a["out"], a["ws"],
                                  a["ws_bytes"], None)


@pytest.mark.parametrize("kw,code", [
    (dict(q=None), E_ARG), (dict(out=None), E_ARG), (dict(clen=None), E_ARG), (dict(batch=0), E_ARG),
    (dict(batch=65536), E_ARG), (dict(n=0), E_ARG), (dict(n=1025), E_ARG), (dict(max_len=-1), E_ARG),
    (dict(max_len=129), E_ARG), (dict(splits=-1), E_ARG), (dict(splits=65536), E_ARG), (dict(scale=0.0), E_ARG),
    (dict(scale=float("nan")), E_ARG), (dict(scale=float("inf")), E_ARG), (dict(hq=5), E_ARG), (dict(hq=6), E_UNS),
    (dict(ms=-1), E_ARG), (dict(ms=1 << 41), E_ARG), (dict(q=at(8) + 8), E_ARG), (dict(out=at(11) + 2), E_ARG),
    (dict(mask=at(10) + 2), E_ARG), (dict(of=at(12) + 2), E_ARG), (dict(splits=2), E_WS),
    (dict(splits=2, ws=at(13), ws_bytes=64), E_WS), (dict(splits=2, ws=at(13) + 4, ws_bytes=1 << 20), E_WS)])
def test_tree_rejects(kw, code):
    assert tree(**kw) == code


@pytest.mark.parametrize("kw", [
    dict(out=at(8)), dict(out=FAKE), dict(out=at(10)), dict(out=at(9)), dict(out=at(2)), dict(of=at(11)),
    dict(splits=2, ws=at(8), ws_bytes=1 << 20), dict(splits=2, ws=at(11), ws_bytes=1 << 20)])
def test_tree_rejects_overlaps(kw):
    assert tree(**kw) == E_ALIAS


def test_tree_valid_calls_reach_the_device():
    assert tree() == E_HIP
    assert tree(mask=None, ms=0) == E_HIP and tree(ms=0) == E_HIP and tree(of=at(12)) == E_HIP
    need = skv.speechkv_tree_workspace_bytes(2, 5, 4, 2, 64, 100, 3)
    assert need > 0 and tree(splits=3, ws=at(13), ws_bytes=need) == E_HIP
    assert tree(splits=3, ws=at(13), ws_bytes=need - 1) == E_WS
    assert tree(max_len=128) == E_HIP and tree(max_len=0) == E_HIP


def test_tree_rejects_an_oversized_grid():
    huge = dict(batch=1000, splits=65535, ws=at(64), ws_bytes=1 << 46, q=1 << 50, out=1 << 51, mask=None)
    assert tree(**huge) == E_UNS
    assert tree(**dict(huge, splits=8000)) == E_HIP  # (2 x 1000 x 8000 blocks: the ranges do not meet)


def test_tree_rejects_a_merge_the_device_cannot_count():
    # 1024 x 480000 rows of 64 elements: 30 million blocks of 16 rows to merge, 8
    # million of 128 rows to attend
    wide = dict(c=cache(num_kv_heads=60000, num_pages=1), batch=1, n=1024, hq=480000, mask=None, ws=at(1 << 21), ws_bytes=1 << 40,
                q=1 << 50, out=1 << 51, clen=1 << 52)
    assert tree(splits=2, **wide) == E_UNS
    assert tree(splits=1, **wide) != E_UNS


def test_tree_rejects_caches_whose_keys_it_cannot_count():
    c = cache(page_size=256, max_pages_per_seq=8388607)
    far = dict(c=c, clen=1 << 50, q=1 << 51, out=1 << 52, mask=None)
    assert tree(max_len=2**31 - 8191, **far) == E_UNS
    assert tree(max_len=2**31 - 8192, **far) == E_HIP


def test_tree_sizes():
    split, ws = skv.speechkv_tree_num_splits, skv.speechkv_tree_workspace_bytes
    BF, F32 = torch.bfloat16, torch.float32
    for bad in ((0, 1, 2, 2, 64, 5), (1, 0, 2, 2, 64, 5), (1, 1025, 2, 2, 64, 5), (1, 1, 3, 2, 64, 5),
                (1, 1, 2, 0, 64, 5), (1, 1, 2, 2, 64, -1), (1, 1, 0, 2, 64, 5), (1, 1, 2, 2, 32, 5)):
        assert split(*bad[:5], BF, bad[5]) == -1
        assert ws(*bad) == 0
    assert split(1, 1, 2, 2, 64, torch.float16, 5) == -1
    assert ws(2, 5, 4, 2, 64, 100, -1) == 0 and ws(2, 5, 4, 2, 64, 100, 1) == 0
    for B in (1, 2, 16, 64):
        for n in (1, 8, 33, 256, 1024):
            for D in (64, 128):
                for L in (0, 1, 100, 2000, 7788, 65536):
                    counts = [split(B, n, 16, 8, D, dt, L) for dt in (BF, F32)]
                    assert all(1 <= s <= 32 and s <= (L + n + 31) // 32 for s in counts)
                    assert ws(B, n, 16, 8, D, L) == ws(B, n, 16, 8, D, L, max(counts))
                    for s in counts:
                        assert s == 1 or ws(B, n, 16, 8, D, L, s) >= B * n * 16 * s * (D + 2) * 4
    assert split(1, 8, 16, 8, 128, BF, 166) == 1 and split(64, 16, 16, 8, 128, BF, 846) == 1
    assert split(1, 8, 16, 8, 128, BF, 7692) > 4


# ------------------------------------------------------------------- commit

def layer(i=0, clen=None, out=None, **kw):
    c = cache(k_pages=at(16 + 8 * i), v_pages=at(17 + 8 * i), block_table=at(18 + 8 * i), **kw)
    return skv._LayerCache(c, at(19 + 8 * i) if clen is None else clen, out)


def commit(layers=None, **kw):
    a = dict(batch=2, path=at(8), m=3, plen=at(9), n=5)
    a.update(kw)
    layers = [layer()] if layers is None else layers
    arr = (skv._LayerCache * max(1, len(layers)))(*layers)
    return lib.speechkv_tree_commit(ctypes.byref(arr), a.get("count", len(layers)), a["batch"], a["path"], a["m"],
                                    a["plen"], a["n"], None)


@pytest.mark.parametrize("kw,code", [
    (dict(path=None), E_ARG), (dict(plen=None), E_ARG), (dict(batch=0), E_ARG), (dict(batch=65536), E_ARG),
    (dict(m=0), E_ARG), (dict(m=6), E_ARG), (dict(n=0), E_ARG), (dict(n=1025, m=1), E_ARG),
    (dict(count=0), E_ARG), (dict(count=257), E_ARG), (dict(count=-1), E_ARG), (dict(path=at(8) + 2), E_ARG)])
def test_commit_rejects(kw, code):
    assert commit(**kw) == code
    assert lib.speechkv_tree_commit(None, 1, 1, at(8), 1, at(9), 1, None) == E_ARG


@pytest.mark.parametrize("layers,code", [
    ([layer(clen=0)], E_ARG), ([layer(head_dim=32)], E_UNS), ([layer(page_size=12)], E_UNS),
    ([layer(), layer(1, head_dim=128)], E_ARG), ([layer(), layer(1, num_kv_heads=4)], E_ARG),
    ([layer(), layer(1, dtype=skv.DTYPE_F32)], E_ARG), ([layer(out=at(19) + 2)], E_ARG),
    ([layer(out=at(19))], E_ALIAS), ([layer(out=at(8))], E_ALIAS), ([layer(out=at(16) + 4)], E_ALIAS),
    ([layer(out=at(20)), layer(1, out=at(20) + 4)], E_ALIAS), ([layer(), layer(1, clen=at(16) + 4)], E_ALIAS),
    ([layer(out=at(27)), layer(1)], E_ALIAS), ([layer(out=at(24) + 8), layer(1)], E_ALIAS)])
def test_commit_rejects_layers(layers, code):
    assert commit(layers) == code


def test_commit_valid_calls_reach_the_device():
    assert commit() == E_HIP
    assert commit([layer(out=at(20)), layer(1, out=at(28), page_size=64, max_pages_per_seq=3)]) == E_HIP
    shared = layer(1)
    shared.cache.k_pages, shared.cache.v_pages = at(16), at(17)
    assert commit([layer(), shared]) == E_HIP  # layers of one pool


# ------------------------------------------------------------------ binding

def host():
    pages = torch.zeros(8, 2, 16, 64, dtype=torch.bfloat16)
    i32 = lambda *s: torch.zeros(*s, dtype=torch.int32)  # noqa: E731
    return dict(cache=skv.PagedKV(pages, pages.clone(), i32(2, 4)), lens=i32(2), i32=i32,
                k=torch.zeros(2, 3, 2, 64, dtype=torch.bfloat16), q=torch.zeros(2, 3, 4, 64, dtype=torch.bfloat16))


def test_layer_packing_fills_its_c_structure():
    x = host()
    out = x["i32"](2)
    s = skv.CacheStack([x["cache"]] * 2, [x["lens"]] * 2, [out, None])
    assert len(s._packed) == 2 * ctypes.sizeof(skv._LayerCache) and (s.num_layers, s.batch) == (2, 2)
    a, b = (skv._LayerCache * 2).from_buffer_copy(s._packed)
    assert a.cache.k_pages == x["cache"].k_pages.data_ptr() and a.cache.dtype == skv.DTYPE_BF16
    assert a.cache_len == x["lens"].data_ptr() and a.cache_len_out == out.data_ptr() and b.cache_len_out is None


@pytest.mark.parametrize("kw", [
    dict(v=torch.zeros(2, 3, 2, 64)), dict(v=torch.zeros(2, 3, 1, 64, dtype=torch.bfloat16)),
    dict(k=torch.zeros(2, 3, 2, 128, dtype=torch.bfloat16)[..., ::2]), dict(q_out=None),
    dict(q_out=torch.zeros(2, 3, 4, 64)), dict(q=torch.zeros(2, 2, 4, 64, dtype=torch.bfloat16)),
    dict(cache_len=torch.zeros(2)), dict(cache_len=torch.zeros(3, dtype=torch.int32)),
    dict(new_len=torch.zeros(2, dtype=torch.int64)), dict(cache_len_out=torch.zeros(4, dtype=torch.int32)[::2]),
    dict(positions=None), dict(positions=torch.zeros(2, 4, dtype=torch.int32)),
    dict(positions=torch.zeros(2, 3)), dict(inv_freq=torch.zeros(8, dtype=torch.float64))])
def test_binding_refuses_append(kw):
    x = host()
    a = dict(k=x["k"], v=x["k"].clone(), cache=x["cache"], cache_len=x["lens"], positions=x["i32"](2, 3),
             inv_freq=torch.zeros(32), q=x["q"], q_out=x["q"].clone(), stream=0)
    a.update(kw)
    with pytest.raises(ValueError):
        skv.speechkv_append_kv(**a)


@pytest.mark.parametrize("kw", [
    dict(out=torch.zeros(2, 3, 4, 64)), dict(out=torch.zeros(2, 4, 3, 64, dtype=torch.bfloat16).transpose(1, 2)),
    dict(q=torch.zeros(1, 3, 4, 64, dtype=torch.bfloat16)), dict(tree_mask=torch.zeros(3, 3, dtype=torch.int32)),
    dict(tree_mask=torch.zeros(2, 3, 1)), dict(tree_mask=torch.zeros(3, 3, 1, dtype=torch.int32)),
    dict(cache_len=torch.zeros(2, dtype=torch.int64)), dict(num_nodes=torch.zeros(1, dtype=torch.int32))])
def test_binding_refuses_tree(kw):
    x = host()
    a = dict(q=x["q"], cache=x["cache"], cache_len=x["lens"], max_cache_len=5, out=x["q"].clone(), stream=0)
    a.update(kw)
    with pytest.raises(ValueError):
        skv.speechkv_tree_attn(**a)


def test_binding_refuses_other_descriptions_for_a_cache():
    x = host()
    spans = skv.Spans(x["lens"], x["lens"], x["lens"], 0, 8)
    with pytest.raises(TypeError):
        skv.speechkv_append_kv(x["k"], x["k"].clone(), spans, x["lens"], stream=0)
    with pytest.raises(TypeError):
        skv.speechkv_tree_attn(x["q"], spans, x["lens"], 5, x["q"].clone(), stream=0)
    with pytest.raises(TypeError):
        skv.CacheStack([spans], [x["lens"]])


def test_binding_refuses_counts_the_library_cannot_hold():
    x = host()
    for bound in (2 ** 31, 2 ** 32 + 5, -1):
        with pytest.raises(skv.SpeechKVError) as e:
            skv.speechkv_tree_attn(x["q"], x["cache"], x["lens"], bound, x["q"].clone(), stream=0)
        assert e.value.status == E_ARG
        with pytest.raises(skv.SpeechKVError) as e:
            skv.speechkv_tree_commit(skv.CacheStack([x["cache"]], [x["lens"]]), x["i32"](2, 1), x["lens"].clone(),
                                     bound, stream=0)
        assert e.value.status == E_ARG


def test_binding_refuses_commit():
    x = host()
    stack = skv.CacheStack([x["cache"]], [x["lens"]])
    with pytest.raises(TypeError):
        skv.speechkv_tree_commit(x["cache"], x["i32"](2, 1), x["lens"], 4, stream=0)
    for path, plen in ((x["i32"](2), x["i32"](2)), (x["i32"](3, 1), x["i32"](2)), (x["i32"](2, 1), x["i32"](3)),
                       (torch.zeros(2, 1), x["i32"](2))):
        with pytest.raises(ValueError):
            skv.speechkv_tree_commit(stack, path, plen, 4, stream=0)
    for args in (([x["cache"]], []), ([x["cache"]], [x["i32"](3)]), ([x["cache"]], [torch.zeros(2)]),
                 ([x["cache"]], [x["lens"]], [x["lens"], None])):
        with pytest.raises(ValueError):
            skv.CacheStack(*args)
    with pytest.raises(skv.SpeechKVError):
        skv.speechkv_tree_commit(skv.CacheStack([], []), x["i32"](0, 1), x["i32"](0), 4, stream=0)


def test_tree_mask_words():
    m = skv.tree_mask([-1, 0, 0, 1], device="cpu")
    assert m.tolist() == [[1], [3], [5], [11]]
    chain = skv.tree_mask([list(range(-1, 39))] * 2, device="cpu")
    assert chain.shape == (2, 40, 2) and chain[1, 31].tolist() == [-1, 0] and chain[0, 32].tolist() == [-1, 1]
    for bad in ([0], [-1, 1], [-1, -2], [[-1], [-1, 0]]):
        with pytest.raises(ValueError):
            skv.tree_mask(bad, device="cpu")
