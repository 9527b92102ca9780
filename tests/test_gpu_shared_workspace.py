"""speechkv_shared_attn with less workspace than its best plan wants, on the GPU
against the 64-bit form: right values, nothing written behind it."""
import pytest
import torch

from gpu_case import guarded
from paper_2607_06827_amd import speechkv as skv
from test_gpu_draft import i32
from test_gpu_shared import DEV, F32, Shared

pytestmark = [pytest.mark.gpu,
              pytest.mark.skipif(not torch.cuda.is_available(), reason="needs a GPU")]


@pytest.mark.parametrize("case", [0, 3, 4, 8, 10])
def test_any_workspace_gives_the_same_attention(case):
    x = Shared(case)
    bound, n = (max(x.prefix), max(x.own)), len(x.prefix)
    best = skv.speechkv_shared_workspace_bytes(x.B, n, x.most, x.Hq, x.Hkv, x.D, *bound)
    a_part = x.B * x.Hq * (x.D + 2) * 4
    assert best >= 2 * a_part
    one = None
    for room in sorted({2 * a_part, 3 * a_part, 3 * a_part + 32, 5 * a_part, best, 40 * a_part}):
        out, rows = guarded(x.q.shape, x.dt, DEV)
        lse, sums = guarded((x.B, x.Hq), F32, DEV)
        ws, behind = guarded((room // 4,), F32, DEV)
        skv.speechkv_shared_attn(x.q, x.pc, i32(x.prefix), bound[0], i32(x.start), x.most, x.oc, i32(x.own), bound[1], out,
                                 lse=lse, workspace=ws)
        torch.cuda.synchronize()
        rows(f"out, {room} bytes")
        sums(f"lse, {room} bytes")
        behind(f"workspace, {room} bytes")
        x.check(out, lse, f"{room} bytes")
        # the least is one range of each, as with one given split where the own
        # entries are one range too
        one = out if room == 2 * a_part else one
    if skv.speechkv_shared_workspace_bytes(x.B, n, x.most, x.Hq, x.Hkv, x.D, *bound, 1) == 2 * a_part:
        given, _ = x.run(splits=1)
        assert torch.equal(given, one)


def test_a_buffer_of_the_largest_step_serves_a_decoding_loop():
    """One buffer, sized once at the limit of the own entries, for every step's
    bound."""
    x = Shared(10)
    limit = x.oc.block_table.shape[1] * x.oc.k_pages.shape[2]
    prefix = max(x.prefix)
    size = skv.speechkv_shared_workspace_bytes(x.B, 1, x.B, x.Hq, x.Hkv, x.D, prefix, limit)
    ws, behind = guarded((size // 4,), F32, DEV)
    keep = x.own
    for step in (1, 64, 128, 500, limit):
        x.own = [min(n, step) for n in keep]
        out, lse = torch.empty_like(x.q), torch.empty(x.B, x.Hq, device=DEV)
        skv.speechkv_shared_attn(x.q, x.pc, i32(x.prefix), prefix, i32(x.start), x.B, x.oc, i32(x.own), step, out, lse=lse,
                                 workspace=ws)
        torch.cuda.synchronize()
        behind(f"workspace, step {step}")
        x.check(out, lse, step)
