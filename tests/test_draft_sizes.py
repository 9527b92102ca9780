"""Sizes that the public limits, the host layer and the kernels of the steps of
several new tokens share: one that is changed alone does not compile (CPU)."""
import os
import shutil
import subprocess

import pytest

from paper_2607_06827_amd import build

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
NODES = ("include/speechkv_draft.h", "#define SPEECHKV_MAX_TREE_NODES 1024", "#define SPEECHKV_MAX_TREE_NODES 2048")
KEYS = ("paper_2607_06827_amd/csrc/kernels_draft.hpp", "kTreeKeys = 32;", "kTreeKeys = 64;")
LAYERS = ("paper_2607_06827_amd/csrc/kernels_draft.hpp", "kCommitLayers = 32;", "kCommitLayers = 128;")


@pytest.mark.skipif(not os.path.exists(build.HIPCC), reason="needs hipcc")
@pytest.mark.parametrize("change,source,compiles", [
    (None, "api_draft.hip", True), (None, "tree_attn.hip", True), (None, "tree_commit.hip", True),
    (NODES, "api_draft.hip", False),   # mask rows and paths in LDS
    (KEYS, "tree_attn.hip", False),    # the tile that the host cuts splits by
    (LAYERS, "tree_commit.hip", False)])  # kernel arguments
def test_sizes_agree(tmp_path, change, source, compiles):
    for d in ("include", "paper_2607_06827_amd/csrc"):
        shutil.copytree(os.path.join(ROOT, d), tmp_path / d)
    if change:
        path, old, new = change
        text = (tmp_path / path).read_text()
        assert text.count(old) == 1
        (tmp_path / path).write_text(text.replace(old, new))
    flags = [f for f in build.DEVICE_FLAGS if f not in ("-mllvm", "-amdgpu-mfma-vgpr-form")]
    r = subprocess.run([build.HIPCC, *flags, "--cuda-host-only", "-fsyntax-only",
                        str(tmp_path / "paper_2607_06827_amd/csrc" / source)],
                       capture_output=True, text=True, timeout=300)
    assert (r.returncode == 0) == compiles, r.stderr
    assert compiles or "static assertion failed" in r.stderr, r.stderr
