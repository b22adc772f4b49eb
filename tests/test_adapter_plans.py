"""The plans of products with adapters, the library's own host arithmetic, swept on the CPU by small drivers linked
to it."""
import shutil
import subprocess

import pytest

from tests import adapter_cases
from tests.test_gated_launches import compile_driver

pytestmark = pytest.mark.skipif(shutil.which("g++") is None, reason="needs g++")


def test_tiles_that_adapters_are_built_for(tmp_path):
    res = subprocess.run([compile_driver("adapter_plans_driver", tmp_path)], capture_output=True, text=True)
    assert res.returncode == 0, res.stdout + res.stderr
    t16, t64, t64x128, t128, t128x256, t256 = map(int, res.stdout.split())
    assert min(t16, t64, t64x128, t128x256) > 100 and t128 == t256 == 0


def test_the_cases_reach_every_path(tmp_path):
    exe = compile_driver("adapter_paths_driver", tmp_path)
    there = set().union(*adapter_cases.paths(exe, adapter_cases.SWEEP))
    reached = set().union(*adapter_cases.paths(exe, adapter_cases.CASES))
    assert there <= reached, sorted(there - reached, key=str)
    # tiles x cut or not x whole ranks or not: bf16 hidden, down and projection, in three tiles; fp32 the same
    assert sum(k[1] != "A x" for k in there) == 2 * 3 * 3 * 2 * 2
