"""The host layers of include/speechkv_norm.h and include/speechkv_shared.h under
AddressSanitizer and UndefinedBehaviorSanitizer (CPU), as tests/test_sanitizers.py
does for that of include/speechkv.h: csrc/api_norm.hip and csrc/api_shared.hip
(host code only) are compiled with both and driven by
tests/sanitize/shared_client.c."""
import os

import pytest
import torch

from test_sanitizers import CLANG, HERE, HIPCC, PKG, ROOT, SAN, run

API = ("api_norm", "api_shared")


@pytest.mark.skipif(not (os.path.exists(HIPCC) and os.path.exists(CLANG)), reason="needs hipcc")
def test_shared_host_layers_under_sanitizers(tmp_path):
    build = os.path.join(PKG, "_build")
    skip = [a + ".hip.o" for a in API] + ["stream_read.hip.o"]
    others = sorted(os.path.join(build, f) for f in os.listdir(build) if f.endswith(".hip.o") and f not in skip) \
        if os.path.isdir(build) else []
    if not others:
        pytest.skip("library objects not built (run __graft_entry__.build())")
    host_san = [x for f in SAN for x in ("-Xarch_host", f)]
    objects = []
    for api in API:
        objects.append(str(tmp_path / (api + ".o")))
        run([HIPCC, "--offload-arch=gfx950", "-O1", "-g", "-std=c++17", "-fPIC", "-Xclang", "-target-feature",
             "-Xclang", "-packed-fp32-ops", *host_san, "-c", os.path.join(PKG, "csrc", api + ".hip"), "-o", objects[-1]])
    lib = tmp_path / "libspeechkv.so"
    run([HIPCC, "--offload-arch=gfx950", "-shared", "-fPIC", "-o", str(lib), *objects, *others])
    exe = tmp_path / "shared_client"
    run([CLANG, "-std=c11", "-O1", "-g", *SAN, f"-I{os.path.join(ROOT, 'include')}",
         os.path.join(HERE, "shared_client.c"), f"-L{tmp_path}", "-lspeechkv",
         f"-Wl,-rpath,{tmp_path}", "-o", str(exe)])
    # valid calls would launch kernels on fake pointers where a GPU exists
    if torch.cuda.device_count() > 0:
        pytest.skip("valid calls would launch kernels on the fake pointers")
    out = run([str(exe), "nodevice"], timeout=300, env=dict(os.environ, ASAN_OPTIONS="detect_leaks=0"))
    assert out.split()[0] == "ok", out
    assert int(out.split()[1]) > 20000
