"""The largest calls of the 8-bit cache and the rotary operator, on the CPU (tests/host_qcache_sizes.cpp): refused before anything is launched where a grid would not hold them."""
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_calls_beyond_a_grid_are_refused(tmp_path):
    gxx = shutil.which("g++")
    if gxx is None or not os.path.exists("/opt/rocm/include/hip/hip_runtime.h"):
        pytest.skip("needs g++ and the HIP headers")
    exe, csrc = str(tmp_path / "host_qcache_sizes"), os.path.join(ROOT, "paper_2511_13587_amd", "csrc")
    cmd = [gxx, "-std=c++17", "-D__HIP_PLATFORM_AMD__", "-I/opt/rocm/include", "-I", os.path.join(ROOT, "include"), "-I", csrc, "-I", os.path.join(ROOT, "tests"), "-g", "-O1", "-w", "-pthread",
           os.path.join(csrc, "vvs_host.cpp"), os.path.join(csrc, "vvs_qcache_host.cpp"), os.path.join(ROOT, "tests", "host_qcache_sizes.cpp"), "-o", exe]
    r = subprocess.run(cmd, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stderr[-3000:]
    r = subprocess.run([exe], capture_output=True, text=True, timeout=100)
    if "no address space" in r.stdout:
        pytest.skip("no address space for the buffers")
    assert r.returncode == 0 and "host qcache sizes ok" in r.stdout, (r.stdout[-2000:], r.stderr[-3000:])
