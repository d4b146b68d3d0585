"""Calls at the documented limits take launches that HIP accepts (fewer than 2^32 threads),
which cover the work once: tests/c/launches.cpp, built here with the library's host code and
no kernels."""
import os
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2609_20359_amd", "csrc")


def test_launches(tmp_path):
    if not os.path.exists("/opt/rocm/include/hip/hip_runtime.h"):
        pytest.skip("no HIP headers")
    exe = str(tmp_path / "launches")
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-D__HIP_PLATFORM_AMD__",
                    "-I/opt/rocm/include", "-I", os.path.join(ROOT, "include"), "-I", CSRC, "-o", exe,
                    os.path.join(ROOT, "tests", "c", "launches.cpp"),
                    os.path.join(CSRC, "flround_layers_api.cpp"),
                    os.path.join(CSRC, "flround_tensors_api.cpp")], check=True)
    r = subprocess.run([exe], capture_output=True, text=True, timeout=60)
    assert r.returncode == 0, r.stdout
    assert "embedding: 1 launches" in r.stdout and "embedding: 4 launches" in r.stdout
    assert "zeros: 1 launches" in r.stdout and "zeros: 8 launches" in r.stdout
