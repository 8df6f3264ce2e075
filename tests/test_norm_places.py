"""Lanes that exchange a head's halves through LDS: each place is stored to by one lane, and read by the lanes that need what is there."""
import os
import shutil
import subprocess

import pytest

from test_host_sanitizers import CSRC, ROOT


@pytest.mark.skipif(shutil.which("g++") is None or not os.path.exists("/opt/rocm/include/hip/hip_runtime.h"), reason="needs g++ and the HIP headers")
def test_every_place_is_one_lanes(tmp_path):
    exe = str(tmp_path / "places")
    res = subprocess.run(["g++", "-std=c++17", "-O2", "-D__HIP_PLATFORM_AMD__", "-I/opt/rocm/include", "-I" + os.path.join(ROOT, "include"), "-I" + CSRC,
                          os.path.join(ROOT, "tests", "norm_places_check.cpp"), "-o", exe], capture_output=True, text=True)
    assert res.returncode == 0, res.stderr[-3000:]
    run = subprocess.run([exe], capture_output=True, text=True)
    assert run.returncode == 0, run.stdout[-2000:]
