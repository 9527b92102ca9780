"""Tests of tests/test_draft_abi.py that pass valid arguments on made-up
addresses must not run where a GPU could launch them, and what they refuse is
tested here in calls of its own, which no machine launches (CPU)."""
import ast
import os
import subprocess
import sys

import pytest

import conftest
from test_abi import cache
from test_draft_abi import E_UNS, E_WS, at, skv, tree

HERE = os.path.dirname(os.path.abspath(__file__))


def test_every_test_that_reaches_the_device_is_named():
    """E_HIP, or anything but a refusal, is expected where the call goes on to the device."""
    found = set()
    for f in ast.parse(open(os.path.join(HERE, "test_draft_abi.py")).read()).body:
        if isinstance(f, ast.FunctionDef) and f.name.startswith("test_"):
            for x in ast.walk(f):
                if isinstance(x, ast.Name) and x.id == "E_HIP" or \
                        isinstance(x, ast.Compare) and any(isinstance(o, ast.NotEq) for o in x.ops):
                    found.add(f.name)
    assert found == set(conftest.VALID_CALLS_ON_FAKE_ADDRESSES["test_draft_abi.py"])


@pytest.mark.parametrize("gpus", [0, 1])
def test_they_are_skipped_where_there_is_a_gpu(tmp_path, gpus):
    """The tests are set up but not run, so that this launches nothing wherever it runs."""
    (tmp_path / "patched.py").write_text(f"import torch\ntorch.cuda.device_count = lambda: {gpus}\n")
    names = conftest.VALID_CALLS_ON_FAKE_ADDRESSES["test_draft_abi.py"]
    ids = [os.path.join(HERE, "test_draft_abi.py") + "::" + n for n in names]
    r = subprocess.run([sys.executable, "-m", "pytest", "-q", "-p", "patched", "-p", "no:cacheprovider",
                        "--setup-plan", *ids],
                       capture_output=True, text=True, timeout=300, cwd=os.path.dirname(HERE),
                       env=dict(os.environ, PYTHONPATH=str(tmp_path)))
    assert r.returncode == 0, r.stdout + r.stderr
    assert (f"{len(names)} skipped" in r.stdout) == bool(gpus), r.stdout


def test_tree_rejects_an_oversized_grid():
    assert tree(batch=1000, splits=65535, ws=at(64), ws_bytes=1 << 46, q=1 << 50, out=1 << 51, mask=None) == E_UNS


def test_tree_rejects_a_merge_the_device_cannot_count():
    assert tree(c=cache(num_kv_heads=60000, num_pages=1), batch=1, n=1024, hq=480000, mask=None, ws=at(1 << 21),
                ws_bytes=1 << 40, q=1 << 50, out=1 << 51, clen=1 << 52, splits=2) == E_UNS


def test_tree_rejects_caches_whose_keys_it_cannot_count():
    assert tree(c=cache(page_size=256, max_pages_per_seq=8388607), clen=1 << 50, q=1 << 51, out=1 << 52, mask=None,
                max_len=2**31 - 8191) == E_UNS


def test_tree_rejects_a_workspace_that_is_one_byte_short():
    need = skv.speechkv_tree_workspace_bytes(2, 5, 4, 2, 64, 100, 3)
    assert need > 0 and tree(splits=3, ws=at(13), ws_bytes=need - 1) == E_WS
