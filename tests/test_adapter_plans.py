"""The plans of products with adapters, the library's own host arithmetic, swept on the CPU by small drivers linked
to it."""
import shutil
import subprocess

import pytest

from tests.test_gated_launches import compile_driver

pytestmark = pytest.mark.skipif(shutil.which("g++") is None, reason="needs g++")


def test_tiles_that_adapters_are_built_for(tmp_path):
    res = subprocess.run([compile_driver("adapter_plans_driver", tmp_path)], capture_output=True, text=True)
    assert res.returncode == 0, res.stdout + res.stderr
    t16, t64, t64x128, t128, t128x256, t256 = map(int, res.stdout.split())
    assert min(t16, t64, t64x128, t128x256) > 100 and t128 == t256 == 0
