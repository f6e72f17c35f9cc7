"""The workspaces of the experts' blocks, and weights that end with a page of memory, without a GPU: experts_plan.cpp built for
the host and driven by tests/sanitize/experts_pages_driver.cpp."""
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
SAN = os.path.join(ROOT, "tests", "sanitize")


def test_workspaces_and_page_ends(tmp_path):
    if shutil.which("g++") is None:
        pytest.skip("no host compiler")
    exe = str(tmp_path / "driver")
    r = subprocess.run(["g++", "-std=c++17", "-O1", "-g", "-D__HIP_PLATFORM_AMD__", "-I", SAN, "-I", "/opt/rocm/include", "-I",
                        os.path.join(ROOT, "include"), os.path.join(ROOT, "paper_2602_21466_amd", "csrc", "experts_plan.cpp"),
                        os.path.join(SAN, "experts_pages_driver.cpp"), "-o", exe], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-3000:]
    r = subprocess.run([exe], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and "workspaces OK" in r.stdout, (r.returncode, r.stdout[-3000:], r.stderr[-2000:])
