"""The host side of the gradient and cache calls (bwd_api.cpp, cache_api.cpp) under
AddressSanitizer and UndefinedBehaviorSanitizer, on the CPU: random sizes, for which what
reaches the launchers has to lie inside the workspace asked for, and refusals
(tests/asan/ops_errors.cpp)."""
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2608_10519_amd", "csrc")
HERE = os.path.join(ROOT, "tests", "asan")


def test_host_side_of_gradients_and_cache_under_sanitizers(tmp_path):
    if shutil.which("g++") is None or not os.path.isdir("/opt/rocm/include"):
        pytest.skip("g++ or the ROCm headers are not available")
    exe = str(tmp_path / "ops_errors")
    src = [os.path.join(CSRC, f) for f in ("host_api.cpp", "bwd_api.cpp", "cache_api.cpp")]
    src += [os.path.join(HERE, f) for f in ("launch_stubs.cpp", "ops_errors.cpp")]
    cmd = ["g++", "-std=c++17", "-O1", "-g", "-fno-omit-frame-pointer", "-fsanitize=address,undefined",
           "-fno-sanitize-recover=undefined", "-D__HIP_PLATFORM_AMD__", "-I/opt/rocm/include", *src,
           "-L/opt/rocm/lib", "-lamdhip64", "-Wl,-rpath,/opt/rocm/lib", "-o", exe]
    b = subprocess.run(cmd, capture_output=True, text=True)
    assert b.returncode == 0, b.stderr[-3000:]
    # a library preloaded into every process would precede the sanitizer's runtime; that order is allowed
    env = dict(os.environ, ASAN_OPTIONS="detect_leaks=1:abort_on_error=0:exitcode=99:verify_asan_link_order=0",
               UBSAN_OPTIONS="print_stacktrace=1:halt_on_error=1")
    r = subprocess.run([exe], capture_output=True, text=True, env=env, timeout=120)
    assert r.returncode == 0, (r.stdout + r.stderr)[-4000:]
    assert " 0 failed" in r.stdout and "checks passed" in r.stdout, r.stdout
