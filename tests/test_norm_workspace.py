"""The workspace of speechkv_norm_rope_bwd: one sized for a program's longest
batch is enough for its shorter ones."""
import pytest

from paper_2607_06827_amd import speechkv as skv
from test_abi import NO_GPU
from test_draft_abi import E_HIP, E_WS, at
from test_norm_abi import bwd, heads

need = skv.speechkv_norm_rope_bwd_workspace_bytes
HEADS = [(64, 8, 64), (16, 8, 128), (1, 1, 128), (2, 1, 64), (16, 0, 128), (0, 5, 64), (160, 3, 128)]
LONGER = [(1, 4096), (1, 16384), (2, 2048), (8, 2048), (64, 2000), (65535, 255)]


def call(batch, rows, hq, hk, D, ws_bytes):
    def view(i, h):
        return heads(i, h, batch, rows, D, data=i << 50) if h else None
    q, k = [view(8 + i, hq) for i in range(3)], [view(16 + i, hk) for i in range(3)]
    return bwd(q=q[0], dyq=q[1], dq=q[2], k=k[0], dyk=k[1], dk=k[2], batch=batch, rows=rows, row_len=None, D=D,
               rope=None, dgq=at(46) if hq else None, dgk=at(47) if hk else None, ws_bytes=ws_bytes)


@pytest.mark.parametrize("hq,hk,D", HEADS)
def test_the_size_does_not_fall_as_rows_or_sequences_grow(hq, hk, D):
    for n in list(range(1, 300)) + list(range(300, 40000, 7)) + [4095, 4096, 4097, 8191, 8192, 16383, 16384, 65536, 131072]:
        size = need(1, n, hq, hk, D)
        assert size >= need(1, max(n - 1, 1), hq, hk, D) and size % (4 * D) == 0 and 0 < size <= 2050 * 4 * D
    for rows in (1, 37, 300, 2048):
        sizes = [need(b, rows, hq, hk, D) for b in range(1, 200)]
        assert sizes == sorted(sizes)


@NO_GPU
@pytest.mark.parametrize("hq,hk,D", HEADS)
@pytest.mark.parametrize("batch,rows", LONGER)
def test_a_workspace_for_the_longest_batch_does_for_shorter_ones(batch, rows, hq, hk, D):
    room = need(batch, rows, hq, hk, D)
    for b, n in ((batch, rows), (batch, rows - 1), (batch, rows // 2), (max(batch - 1, 1), rows), (1, rows), (1, 1),
                 (batch, 1), (max(batch // 3, 1), max(rows // 3, 1))):
        assert call(b, n, hq, hk, D, room) == E_HIP, (b, n)
        assert call(b, n, hq, hk, D, need(b, n, hq, hk, D) - 1) == E_WS
