"""The plans of the gated block's products (tiles, shares, room for their sums): the library's own host
arithmetic, swept on the CPU by a small driver linked to it."""
import os
import shutil
import subprocess

import pytest

from paper_2609_31975_amd import build, ffn

HERE = os.path.dirname(os.path.abspath(__file__))


@pytest.mark.skipif(shutil.which("g++") is None, reason="needs g++")
def test_every_plan_fits(tmp_path):
    ffn.lib()
    exe = str(tmp_path / "gated_plans")
    subprocess.run(["g++", "-O2", "-std=c++17", "-D__HIP_PLATFORM_AMD__", "-I", os.path.join(build.PKG, "csrc"), "-I",
                    "/opt/rocm/include", os.path.join(HERE, "gated_plans_driver.cpp"), build.LIB, "-L/opt/rocm/lib",
                    "-lamdhip64", f"-Wl,-rpath,{build.PKG}", "-Wl,-rpath,/opt/rocm/lib", "-o", exe], check=True)
    res = subprocess.run([exe], capture_output=True, text=True)
    assert res.returncode == 0, res.stdout + res.stderr
    plans, cut = map(int, res.stdout.split())
    assert plans > 100000 and cut > 10000  # both kinds were reached
