"""The checks of linear attention, the norm and the choice of tokens under AddressSanitizer and UndefinedBehaviorSanitizer (host
code only)."""
import os
import shutil

import pytest

from test_host_sanitizers import ENV, HOST, ROOT, run


def test_block_api_host_logic_under_asan_ubsan(tmp_path):
    hipcc = "/opt/rocm/bin/hipcc" if os.path.exists("/opt/rocm/bin/hipcc") else shutil.which("hipcc")
    if not hipcc:
        pytest.skip("hipcc not available")
    exe = str(tmp_path / "block_api_selftest")
    csrc = os.path.join(ROOT, "paper_2503_01868_amd", "csrc")
    san = ["-Xarch_host", "-fsanitize=address", "-Xarch_host", "-fsanitize=undefined", "-Xarch_host", "-fno-omit-frame-pointer"]
    build = run([hipcc, "--offload-arch=gfx950", "-O1", "-g", "-std=c++17", "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
                 "-I" + os.path.join(ROOT, "include"), "-I" + csrc] + san + [
                     os.path.join(csrc, "block_api.hip"), "-x", "hip", os.path.join(HOST, "block_api_selftest.cpp"), "-o", exe])
    assert build.returncode == 0, build.stderr[-3000:]
    res = run([exe], env=ENV)
    out = res.stdout + res.stderr
    assert "AddressSanitizer" not in out and "runtime error" not in out, out[-3000:]
    assert "block api selftest: 0 problem(s)" in res.stdout, out[-3000:]
