"""The grids of the gated block's and the adapters' calls over very many tokens: the library's own host arithmetic,
swept on the CPU by a small driver linked to it."""
import os
import shutil
import subprocess

import pytest

from paper_2609_31975_amd import build, ffn

HERE = os.path.dirname(os.path.abspath(__file__))


def compile_driver(name, tmp_path):
    ffn.lib()
    exe = str(tmp_path / name)
    subprocess.run(["g++", "-O2", "-std=c++17", "-D__HIP_PLATFORM_AMD__", "-I", os.path.join(build.PKG, "csrc"), "-I",
                    "/opt/rocm/include", os.path.join(HERE, f"{name}.cpp"), build.LIB, "-L/opt/rocm/lib", "-lamdhip64",
                    f"-Wl,-rpath,{build.PKG}", "-Wl,-rpath,/opt/rocm/lib", "-o", exe], check=True)
    return exe


@pytest.mark.skipif(shutil.which("g++") is None, reason="needs g++")
def test_every_grid_is_one_that_hip_takes(tmp_path):
    res = subprocess.run([compile_driver("gated_launches_driver", tmp_path)], capture_output=True, text=True)
    assert res.returncode == 0, res.stdout + res.stderr
    assert int(res.stdout) > 10000


def test_workspaces_of_the_most_tokens():
    """Up to 2^31 - 1 tokens of one element: sizes go on growing."""
    L = ffn.lib()
    tokens = [1 << 27, (1 << 30) - 1, 1 << 30, (1 << 31) - 256, (1 << 31) - 255, (1 << 31) - 1]
    for wdt in (0, 1):
        for sizes in ([L.ffn_adapter_workspace_bytes(wdt, T, 1, 1, 1) for T in tokens],
                      [L.ffn_gated_workspace_bytes(wdt, T, 1, 1, 1, 0) for T in tokens],
                      [L.ffn_gated_save_bytes(wdt, T, 1) for T in tokens]):
            assert sizes == sorted(sizes) and sizes[0] > 0
