"""The host code of the C entries of low-rank adapters, gradient norms and the
verification of drafts under AddressSanitizer + UndefinedBehaviorSanitizer:
tests/more_operators_host_check.cpp with their three sources (host code
instrumented, device code as usual).  Skipped where a GPU is visible (its calls
with pointers to host memory must end before one) or hipcc is missing."""

import os
import shutil
import subprocess

import pytest

from paper_1903_05133_amd import build
from test_abi_sanitized import CSRC, ROOT, _gpu_visible


@pytest.mark.skipif(_gpu_visible(), reason="its calls end at the missing GPU")
def test_more_operators_host_code_under_sanitizers(tmp_path):
    if not shutil.which(build.hipcc()):
        pytest.skip("hipcc not found")
    exe = str(tmp_path / "more_operators_host_check")
    cmd = [build.hipcc(), "--offload-arch=gfx950", "-O1", "-g", "-std=c++17",
           "-Xarch_host", "-fsanitize=address", "-Xarch_host", "-fsanitize=undefined",
           "-Xarch_host", "-fno-sanitize-recover=undefined",
           "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
           "-I", os.path.join(ROOT, "include"), "-I", CSRC,
           os.path.join(ROOT, "tests", "more_operators_host_check.cpp"), *[os.path.join(CSRC, s) for s in ("k_clip.hip", "k_verify.hip", "k_adapters.hip")],
           "-o", exe]
    res = subprocess.run(cmd, capture_output=True, text=True, timeout=600)
    assert res.returncode == 0, res.stderr[-4000:]
    env = dict(os.environ, ASAN_OPTIONS="detect_leaks=1:halt_on_error=1", UBSAN_OPTIONS="halt_on_error=1")
    run = subprocess.run([exe], capture_output=True, text=True, timeout=300, env=env)
    assert run.returncode == 0, run.stdout[-4000:] + run.stderr[-4000:]
    assert "host checks ok" in run.stdout
