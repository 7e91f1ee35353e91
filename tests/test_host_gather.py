"""Gathers out of a pool in 8 bits over a stand-in for the HIP runtime (tests/host_gather.cpp), compiled for the CPU: what the launch is told."""
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2504_19867_amd", "csrc")


def test_a_gather_knows_its_share(tmp_path):
    gxx = shutil.which("g++")
    if gxx is None or not os.path.isdir("/opt/rocm/include"):
        pytest.skip("needs g++ and the HIP headers")
    exe = str(tmp_path / "host_gather")
    build = subprocess.run([gxx, "-std=c++17", "-O1", "-g", "-D__HIP_PLATFORM_AMD__", "-I/opt/rocm/include", "-I", os.path.join(ROOT, "include"),
                            "-I", CSRC, *[os.path.join(CSRC, f) for f in ("ctx.cpp", "steps.cpp", "pool.cpp", "rope.cpp")],
                            os.path.join(ROOT, "tests", "host_gather.cpp"), "-o", exe, "-lpthread"], capture_output=True, text=True)
    assert build.returncode == 0, build.stderr[-3000:]
    run = subprocess.run([exe], capture_output=True, text=True, timeout=60)
    assert run.returncode == 0 and run.stdout == "ok\n", run.stderr[-2000:]
