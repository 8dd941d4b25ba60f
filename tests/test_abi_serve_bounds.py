"""What the 4-bit cache and eviction entry points hand to their kernels, without a GPU: the host side under
AddressSanitizer and UndefinedBehaviorSanitizer, the launches replaced by stubs that keep the arguments."""
import os
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2606_24957_amd", "csrc")
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")


@pytest.mark.skipif(not os.path.exists(HIPCC), reason="hipcc not available")
def test_bounds_under_asan_and_ubsan(tmp_path):
    exe = str(tmp_path / "abi_serve_bounds")
    # host code only is instrumented (each -fsanitize= behind -Xarch_host)
    cmd = [HIPCC, "--offload-arch=gfx950", "-x", "hip", "-O1", "-g", "-std=c++17", "-fno-omit-frame-pointer",
           "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
           "-Xarch_host", "-fsanitize=address", "-Xarch_host", "-fsanitize=undefined",
           "-Xarch_host", "-fno-sanitize-recover=undefined",
           "-I", os.path.join(ROOT, "include"), "-I", CSRC, os.path.join(CSRC, "api_kv4.hip"),
           os.path.join(ROOT, "tests", "sanitize", "abi_serve_bounds.cpp"), "-o", exe]
    r = subprocess.run(cmd, capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-4000:]
    env = dict(os.environ, ASAN_OPTIONS="detect_leaks=0:abort_on_error=0", UBSAN_OPTIONS="print_stacktrace=1")
    run = subprocess.run([exe], capture_output=True, text=True, env=env, timeout=120)
    out = run.stdout + run.stderr
    assert run.returncode == 0, out[-4000:]
    assert "ok: 0 failed expectations" in out
    for report in ("ERROR: AddressSanitizer", "runtime error:", "ERROR: LeakSanitizer", "UndefinedBehaviorSanitizer"):
        assert report not in out, out[-4000:]
