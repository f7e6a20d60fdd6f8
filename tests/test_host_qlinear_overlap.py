"""Tensors of a linear map that lie over each other or in its own buffers are refused (tests/host_qlinear_overlap.cpp)."""
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_overlaps_are_refused(tmp_path):
    gxx = shutil.which("g++")
    if gxx is None or not os.path.exists("/opt/rocm/include/hip/hip_runtime.h"):
        pytest.skip("needs g++ and the HIP headers")
    exe, csrc = str(tmp_path / "host_qlinear_overlap"), os.path.join(ROOT, "paper_2511_13587_amd", "csrc")
    cmd = [gxx, "-std=c++17", "-D__HIP_PLATFORM_AMD__", "-I/opt/rocm/include", "-I", os.path.join(ROOT, "include"), "-I", csrc, "-O1", "-w",
           os.path.join(csrc, "vvs_qlinear_host.cpp"), os.path.join(ROOT, "tests", "host_qlinear_overlap.cpp"), "-o", exe]
    r = subprocess.run(cmd, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stderr[-3000:]
    r = subprocess.run([exe], capture_output=True, text=True, timeout=60)
    assert r.returncode == 0 and "ok" in r.stdout, (r.stdout, r.stderr)
