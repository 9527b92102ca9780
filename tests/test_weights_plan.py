"""How speechkv_attn_weights cuts a call (csrc/attn_weights.hip), asked of the built
library by a small host program."""
import os
import subprocess

import pytest

from paper_2607_06827_amd import speechkv as skv
from paper_2607_06827_amd.build import CSRC, HIPCC
from test_kernel_resources import kernels
from weights_cases import BF, TWO_STRETCHES, requested_ahead, row_tiles

CLIENT = r"""
#include "kernels_shared.hpp"
#include <stdio.h>
int main() {
  int batch, heads, max_len, tiles, dim, esz;
  while (scanf("%d %d %d %d %d %d", &batch, &heads, &max_len, &tiles, &dim, &esz) == 6) {
    skv::WeightArgs a = {};
    a.batch = batch;
    a.cache.pv.kv_heads = heads;
    a.cache.max_len = max_len;
    a.row_tiles = tiles;
    skv::plan_weights(a, dim, esz);
    printf("%d %d %d\n", a.steps, a.stretches, a.key_blocks);
  }
  return 0;
}
"""


@pytest.fixture(scope="module")
def plan(tmp_path_factory):
    """plan([(batch, KV heads, longest cache, row tiles, head_dim, element bytes)]) ->
    [(steps of a wave, stretches of a block, blocks of a (sequence, KV head))]."""
    if not os.path.exists(HIPCC):
        pytest.skip("needs hipcc")
    at = tmp_path_factory.mktemp("plan")
    (at / "plan.hip").write_text(CLIENT)
    lib = os.path.dirname(skv.LIBRARY_PATH)
    subprocess.run([HIPCC, "--offload-arch=gfx950", "-O1", "-std=c++17", f"-I{CSRC}",
                    str(at / "plan.hip"), "-o", str(at / "plan"), f"-L{lib}", "-lspeechkv", f"-Wl,-rpath,{lib}"], check=True,
                   capture_output=True)

    def ask(calls):
        text = "".join(" ".join(map(str, c)) + "\n" for c in calls)
        out = subprocess.run([str(at / "plan")], input=text, check=True, capture_output=True, text=True).stdout
        return [tuple(map(int, line.split())) for line in out.splitlines()]
    return ask


def test_the_cases_of_two_stretches_take_two(plan):
    got = plan([(len(c[5]), c[3], max(c[5]), row_tiles(c), c[1], 2 if c[0] == BF else 4) for c in TWO_STRETCHES])
    assert len(got) == len(TWO_STRETCHES)
    for c, (steps, stretches, blocks) in zip(TWO_STRETCHES, got):
        keys = 32 if requested_ahead(c) == 16 else 64
        assert stretches == 2 and blocks == -(-max(c[5]) // (2 * keys)), c
        assert row_tiles(c) > requested_ahead(c), c
    assert any(row_tiles(c) % 8 for c in TWO_STRETCHES) and sum(row_tiles(c) > 512 for c in TWO_STRETCHES) >= 2


# bf16 and fp32 rows of 64 and 128 elements: the kernel's name in the library
FEW = {(64, 2): "weights_few_kernelItLi64E", (128, 2): "weights_few_kernelItLi128E",
       (64, 4): "weights_few_kernelIfLi64E", (128, 4): "weights_few_kernelIfLi128E"}
CUS, LDS = 256, 160 * 1024


@pytest.mark.parametrize("dim,esz", list(FEW))
def test_few_rows_spread_over_the_blocks_that_run_at_once(plan, dim, esz):
    """A wave's steps cut the keys for one round of blocks, of as many as a CU's LDS
    holds, or, one a CU, for as few whole rounds as it takes."""
    found = [k for n, k in kernels().items() if FEW[dim, esz] in n]
    assert len(found) == 1
    at_once = CUS * min(LDS // found[0][".group_segment_fixed_size"], 2)
    calls = [(B, H, L, 1, dim, esz) for B in (1, 2, 3, 8, 16, 40) for H in (1, 4, 8) for L in (1, 31, 471, 1600, 7660, 60000)]
    for (B, H, L, *_), (steps, _, blocks) in zip(calls, plan(calls)):
        tiles = -(-L // 32)
        rounds = -(-B * H * tiles // (at_once * 4 * 16)) if at_once == CUS else 1  # of 16 steps a wave at most
        assert 1 <= steps <= 16 and blocks == -(-tiles // (4 * steps))
        assert steps == min(-(-B * H * tiles // (at_once * 4 * rounds)), 16), (B, H, L, steps, rounds)
