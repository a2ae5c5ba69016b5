"""The checks of the single-token step's C entry points built with
AddressSanitizer and UndefinedBehaviorSanitizer (CPU only) and driven over
random, invalid and extreme arguments; launches are replaced by stand-ins that
launch nothing."""
import os
import subprocess

import pytest

from paper_2111_05426_amd import build

HERE = os.path.dirname(os.path.abspath(__file__))
CLANG = "/opt/rocm/llvm/bin/clang++"


@pytest.mark.skipif(not os.path.exists(CLANG), reason="the ROCm clang is not installed")
def test_operators_host_validation_under_sanitizers(tmp_path):
    exe = str(tmp_path / "ops_driver")
    cmd = [CLANG, "-std=c++17", "-O1", "-g", "-D__HIP_PLATFORM_AMD__", "-I", "/opt/rocm/include", "-I", build.INCLUDE,
           "-fsanitize=address,undefined", "-fno-sanitize-recover=all", "-o", exe,
           os.path.join(HERE, "sanitize", "ops_driver.cpp"), os.path.join(build.CSRC, "api_ops.cpp"),
           "-L/opt/rocm/lib", "-lamdhip64", "-Wl,-rpath,/opt/rocm/lib"]
    p = subprocess.run(cmd, capture_output=True, text=True, timeout=600)
    assert p.returncode == 0, p.stderr
    env = dict(os.environ, ASAN_OPTIONS="detect_leaks=0", UBSAN_OPTIONS="print_stacktrace=1")
    p = subprocess.run([exe], capture_output=True, text=True, timeout=600, env=env)
    assert p.returncode == 0 and "runtime error" not in p.stderr and "AddressSanitizer" not in p.stderr, p.stderr
    assert "reached a launch" in p.stdout
