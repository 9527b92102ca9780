"""The host layer of include/speechkv_draft.h under AddressSanitizer and
UndefinedBehaviorSanitizer (CPU), as tests/test_sanitizers.py does for that of
include/speechkv.h: csrc/api_draft.hip (host code only) is compiled with both
and driven by tests/sanitize/draft_client.c."""
import os

import pytest
import torch

from test_sanitizers import CLANG, HERE, HIPCC, PKG, ROOT, SAN, run


@pytest.mark.skipif(not (os.path.exists(HIPCC) and os.path.exists(CLANG)), reason="needs hipcc")
def test_draft_host_layer_under_sanitizers(tmp_path):
    build = os.path.join(PKG, "_build")
    others = sorted(os.path.join(build, f) for f in os.listdir(build)
                    if f.endswith(".hip.o") and f not in ("api_draft.hip.o", "stream_read.hip.o")) \
        if os.path.isdir(build) else []
    if not others:
        pytest.skip("library objects not built (run __graft_entry__.build())")
    api = tmp_path / "api_draft.o"
    host_san = [x for f in SAN for x in ("-Xarch_host", f)]
    run([HIPCC, "--offload-arch=gfx950", "-O1", "-g", "-std=c++17", "-fPIC", "-Xclang", "-target-feature",
         "-Xclang", "-packed-fp32-ops", *host_san, "-c", os.path.join(PKG, "csrc", "api_draft.hip"), "-o", str(api)])
    lib = tmp_path / "libspeechkv.so"
    run([HIPCC, "--offload-arch=gfx950", "-shared", "-fPIC", "-o", str(lib), str(api), *others])
    exe = tmp_path / "draft_client"
    run([CLANG, "-std=c11", "-O1", "-g", *SAN, f"-I{os.path.join(ROOT, 'include')}",
         os.path.join(HERE, "draft_client.c"), f"-L{tmp_path}", "-lspeechkv",
         f"-Wl,-rpath,{tmp_path}", "-o", str(exe)])
    # valid calls would launch kernels on fake pointers where a GPU exists
    args = [] if torch.cuda.device_count() > 0 else ["nodevice"]
    out = run([str(exe), *args], timeout=300, env=dict(os.environ, ASAN_OPTIONS="detect_leaks=0"))
    assert out.split()[0] == "ok", out
    assert int(out.split()[1]) > 3000
