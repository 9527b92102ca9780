"""speechkv_shared_attn that chooses its splits does with any workspace that
holds one range of the prefix and one of the own entries a row: a buffer sized
for a program's largest call is enough for its smaller ones, though their best
plan may want more."""
import pytest
import torch

from paper_2607_06827_amd import speechkv as skv
from test_abi import NO_GPU, cache
from test_draft_abi import E_HIP, E_WS, at
from test_shared_abi import shared

CODES = {skv.DTYPE_BF16: torch.bfloat16, skv.DTYPE_F32: torch.float32}


def call(B, groups, most, Hkv, P, L, ws_bytes, ws=at(1 << 12), dtype=skv.DTYPE_BF16, G=2, splits=0, D=128):
    """One call; the status."""
    kw = dict(num_kv_heads=Hkv, head_dim=D, dtype=dtype, num_pages=512, max_pages_per_seq=1024)
    p = cache(k_pages=1 << 50, v_pages=1 << 51, block_table=1 << 52, **kw)
    c = cache(k_pages=1 << 53, v_pages=1 << 54, block_table=1 << 55, **kw)
    return shared(p=p, c=c, batch=B, hq=G * Hkv, groups=groups, most=most, max_prefix=P, max_len=L, splits=splits,
                  q=1 << 56, out=1 << 57, lse=1 << 58, plen=1 << 59, start=1 << 60, clen=1 << 61, ws=ws, ws_bytes=ws_bytes)


def need(B, groups, most, Hkv, P, L, splits=0, G=2, D=128):
    return skv.speechkv_shared_workspace_bytes(B, groups, most, G * Hkv, Hkv, D, P, L, splits)


def least(B, Hkv, G=2, D=128):
    return B * G * Hkv * 2 * (D + 2) * 4


# (the largest call, a smaller one whose best plan needs more): own entries,
# members of the longest group, the prefix
GROWING = [((64, 1, 64, 8, 7532, 2048), (64, 1, 64, 8, 7532, 128)), ((64, 1, 64, 8, 7532, 2048), (64, 1, 64, 8, 7532, 1)),
           ((8, 1, 8, 8, 7532, 2048), (8, 1, 8, 8, 7532, 128)), ((8, 1, 8, 8, 7532, 2048), (8, 1, 8, 8, 7532, 0)),
           ((64, 1, 64, 8, 1000, 96), (64, 1, 64, 8, 64, 96))]


@NO_GPU
@pytest.mark.parametrize("dtype", list(CODES))
@pytest.mark.parametrize("large,small", GROWING)
def test_a_workspace_for_the_largest_call_does_for_smaller_ones(large, small, dtype):
    room, best = need(*large), need(*small)
    assert room < best
    for x in (large, small):
        assert call(*x, room, dtype=dtype) == E_HIP
        for size in (least(small[0], 8), least(small[0], 8) + 8, best - 4, best, 1 << 40):
            assert call(*x, size, dtype=dtype) == E_HIP, (x, size)


@NO_GPU
def test_the_largest_batch_does_for_every_call():
    """A decoding loop allocates once, for its most questions and entries."""
    for D in (64, 128):
        room = need(48, 6, 48, 4, 7532, 2048, D=D)
        for B in (1, 2, 7, 30, 48):
            for groups, most in ((1, B), (min(B, 6), 1 + B // 6)):
                for P in (0, 1, 126, 1500, 7532):
                    for L in (0, 1, 40, 300, 2048):
                        for dtype in CODES:
                            assert call(B, groups, most, 4, P, L, room, dtype=dtype, D=D) == E_HIP, (B, groups, P, L, D)


def test_less_than_the_least_is_refused():
    for dtype in CODES:
        x = (8, 1, 8, 8, 7532, 128)
        assert call(*x, least(8, 8) - 1, dtype=dtype) == E_WS and call(*x, 0, dtype=dtype) == E_WS
        assert call(*x, 1 << 40, None, dtype) == E_WS
        assert call(*x, 1 << 40, at(1 << 12) + 8, dtype) == E_WS


def test_a_given_split_count_needs_its_size():
    """Refused before anything is launched."""
    for s in (1, 3, 7):
        assert call(8, 1, 8, 8, 7532, 128, least(8, 8) * (s + 1) // 2 - 1, splits=s) == E_WS
        size = need(8, 1, 8, 8, 7532, 128, s)
        assert E_WS in [call(8, 1, 8, 8, 7532, 128, size - 4, dtype=t, splits=s) for t in CODES]


def test_the_size_and_the_count_are_those_of_a_call_with_room():
    """What the helpers say does not follow from any workspace."""
    for x in GROWING[0] + GROWING[2]:
        B, groups, most, Hkv, P, L = x
        counts = [skv.speechkv_shared_num_splits(B, groups, most, 2 * Hkv, Hkv, 128, t, P, L) for t in CODES.values()]
        assert need(*x) >= (max(counts) + 1) * least(B, Hkv) // 2
