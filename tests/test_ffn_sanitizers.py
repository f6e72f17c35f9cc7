"""The feed-forward sublayer's host code under AddressSanitizer and UndefinedBehaviorSanitizer (CPU only).

ffn_plan.cpp is built host-only with g++ against the stand-in for the HIP runtime in tests/sanitize/ and driven by
tests/sanitize/ffn_driver.cpp, whose launchers do on the host what the kernels are asked for, so that workspace layouts,
strides, paddings, parts of k and the order of the launches are held against the definitions in 64 bits.
"""
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
SAN = os.path.join(ROOT, "tests", "sanitize")


def test_host_code_of_the_sublayer(tmp_path):
    if shutil.which("g++") is None:
        pytest.skip("no host compiler")
    flags = ["-std=c++17", "-O1", "-g", "-fno-omit-frame-pointer", "-fsanitize=address,undefined", "-fno-sanitize-recover=all",
             "-D__HIP_PLATFORM_AMD__", "-I", SAN, "-I", "/opt/rocm/include", "-I", os.path.join(ROOT, "include")]
    exe = str(tmp_path / "driver")
    r = subprocess.run(["g++"] + flags + [os.path.join(ROOT, "paper_2602_21466_amd", "csrc", "ffn_plan.cpp"),
                                          os.path.join(SAN, "ffn_driver.cpp"), "-o", exe], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-3000:]
    env = dict(os.environ, ASAN_OPTIONS="detect_leaks=1:abort_on_error=0", UBSAN_OPTIONS="print_stacktrace=1:halt_on_error=1")
    r = subprocess.run([exe], capture_output=True, text=True, timeout=600, env=env)
    assert r.returncode == 0, (r.stdout[-3000:], r.stderr[-4000:])
    assert "sanitized host code OK" in r.stdout
    assert "runtime error" not in r.stderr and "ERROR: AddressSanitizer" not in r.stderr
