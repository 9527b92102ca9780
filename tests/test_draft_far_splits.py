"""Key numbers of speechkv_tree_attn's splits stay in 31 bits (CPU: the calls
are refused before anything is launched, or end for want of a device)."""
import pytest

from test_abi import NO_GPU, cache
from test_draft_abi import E_HIP, E_UNS, at, tree


def far(max_len, splits, n=5):
    c = cache(page_size=256, max_pages_per_seq=8388607)
    return tree(c=c, clen=1 << 50, q=1 << 51, out=1 << 52, mask=None, max_len=max_len, splits=splits, batch=1, n=n,
                ws=at(1 << 12), ws_bytes=1 << 40)


def last_key(max_len, splits, n):
    """Past the last key that a block of the last split works out: the splits are
    cut from the bound in whole tiles of 32 keys, and a block looks 16 steps of
    four tiles ahead."""
    tiles = -(-(max_len + n) // 32)
    return (-(-tiles // splits) * splits + 64) * 32


@pytest.mark.parametrize("max_len,splits,n", [(2**31 - 8192, 65535, 5), (2**31 - 8192, 60001, 1024),
                                              (2**31 - 18192, 65535, 1)])
def test_splits_that_reach_past_31_bits_are_refused(max_len, splits, n):
    assert last_key(max_len, splits, n) > 2**31
    assert far(max_len, splits, n) == E_UNS


@NO_GPU
@pytest.mark.parametrize("max_len,splits,n", [(2**31 - 8192, 1, 1024), (2**31 - 8192, 32, 1024),
                                              (2**31 - 4 * 10**6, 65535, 1024), (7692, 65535, 8)])
def test_others_are_not(max_len, splits, n):
    assert last_key(max_len, splits, n) <= 2**31
    assert far(max_len, splits, n) == E_HIP
