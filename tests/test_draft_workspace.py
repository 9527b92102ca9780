"""speechkv_tree_attn that chooses its splits does with any workspace: one sized
for a program's largest call is enough for its smaller ones, though their best
split count may want more."""
import pytest

from paper_2607_06827_amd import speechkv as skv
from test_abi import NO_GPU, cache
from test_draft_abi import E_HIP, E_WS, at, tree


def call(B, n, Hkv, L, ws_bytes, ws=at(1 << 12), dtype=skv.DTYPE_BF16):
    c = cache(num_kv_heads=Hkv, head_dim=128, dtype=dtype, num_pages=512, max_pages_per_seq=512)
    far = dict(q=1 << 50, out=1 << 51, clen=1 << 52, mask=None)
    return tree(c=c, batch=B, n=n, hq=2 * Hkv, max_len=L, splits=0, ws=ws, ws_bytes=ws_bytes, **far)


# (the largest call, a smaller one whose best split count needs more)
GROWING = [((8, 32, 8, 7999), (8, 32, 8, 7168)), ((16, 32, 8, 2160), (16, 32, 8, 2144)),
           ((4, 1024, 8, 2000), (4, 256, 8, 2000)), ((4, 8, 8, 7700), (3, 8, 8, 7700)),
           ((17, 4, 8, 200), (16, 4, 8, 200))]


def need(B, n, Hkv, L):
    return skv.speechkv_tree_workspace_bytes(B, n, 2 * Hkv, Hkv, 128, L)


@NO_GPU
@pytest.mark.parametrize("dtype", [skv.DTYPE_BF16, skv.DTYPE_F32])
@pytest.mark.parametrize("large,small", GROWING)
def test_a_workspace_for_the_largest_call_does_for_smaller_ones(large, small, dtype):
    assert need(*large) < need(*small)
    room = need(*large)
    assert call(*large, room, dtype=dtype) == E_HIP and call(*small, room, dtype=dtype) == E_HIP
    assert call(*small, 0, None, dtype) == E_HIP and call(*small, 1 << 40, None, dtype) == E_HIP
    assert call(*small, 16, dtype=dtype) == E_HIP and call(*small, need(*small) - 1, dtype=dtype) == E_HIP


@NO_GPU
def test_any_size_does_for_any_call():
    for B in (1, 3, 16):
        for n in (1, 40, 1024):
            for L in (0, 300, 8000):
                for room in (0, 1 << 12, 1 << 20, 1 << 25):
                    for dtype in (skv.DTYPE_BF16, skv.DTYPE_F32):
                        assert call(B, n, 4, L, room, dtype=dtype) == E_HIP, (B, n, L, room)


def test_a_given_split_count_needs_its_size():
    """Refused before anything is launched."""
    c = dict(c=cache(), batch=2, n=5, hq=4, max_len=100)
    for s in (2, 3, 7):
        size = skv.speechkv_tree_workspace_bytes(2, 5, 4, 2, 64, 100, s)
        assert tree(splits=s, ws=at(13), ws_bytes=size - 1, **c) == E_WS
        assert tree(splits=s, ws=None, ws_bytes=size, **c) == E_WS


def test_an_unaligned_workspace_is_refused_where_it_would_be_used():
    assert call(1, 8, 8, 7692, 1 << 24, ws=at(1 << 12) + 8) == E_WS
