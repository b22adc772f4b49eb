"""The norms' launches up to the most rows that a call takes: the library's own host arithmetic, swept on the CPU by a small
driver linked to it, and the workspace that follows from it."""
import random
import shutil
import subprocess

import pytest

from paper_2609_31975_amd import ffn
from tests import norm_chains
from tests.test_gated_launches import compile_driver

MOST = (1 << 31) - 1        # T d of a call


def sizes():
    rng = random.Random(7)
    out = [(MOST // d - i, d) for d in (1, 2, 3, 64, 512, 513, 1024, 1025, 2048, 2049, 4096, 4097, 8192, 8193, 16384) for i in (0, 1, 2, 3)]
    for _ in range(20000):
        d = int(2 ** rng.uniform(0, 14))
        out.append((int(2 ** rng.uniform(0, 31)) % (MOST // d) + 1, d))
    return out


@pytest.mark.skipif(shutil.which("g++") is None, reason="needs g++")
def test_every_row_has_a_group_and_every_grid_is_one_that_hip_takes(tmp_path):
    cases = sizes()
    res = subprocess.run([compile_driver("norm_plans_driver", tmp_path)], input="".join(f"{T} {d}\n" for T, d in cases),
                         capture_output=True, text=True, check=True)
    lines = [tuple(map(int, line.split())) for line in res.stdout.splitlines()]
    assert len(lines) == len(cases)
    for (T, d), (tpr, ept, blocks, b_tpr, b_ept, groups) in zip(cases, lines):
        what = (T, d, tpr, ept, blocks, b_tpr, b_ept, groups)
        assert (tpr, ept) in {(64, 8), (64, 16), (256, 8), (256, 16), (512, 16), (1024, 16)} and tpr * ept >= d, what
        assert (b_tpr, b_ept) in {(64, 8), (256, 8), (512, 8), (1024, 8), (1024, 16)} and b_tpr * b_ept >= d, what
        rows = 4 if tpr == 64 else 1
        assert 1 <= blocks <= 1 << 20 and (blocks - 1) * rows < T, what
        assert blocks == 1 << 20 or blocks * rows >= T, what
        assert blocks * max(tpr, 256) < 1 << 32, what
        assert 1 <= groups <= 2048 and groups % (4 if b_tpr == 64 else 1) == 0 and groups < T + 4, what
        assert groups == norm_chains.groups(T, d), what


def test_workspaces_of_the_most_rows():
    """Sizes go on growing up to the most rows, and stay what a few thousand rows' partial sums take."""
    L = ffn.lib()
    for d in (1, 2, 33, 512, 513, 2048, 2049, 4096, 4097, 8192, 16384):
        most = MOST // d
        got = [L.ffn_norm_workspace_bytes(T, d) for T in (1, 2, most // 2, most - 3, most - 2, most - 1, most)]
        assert got == sorted(got) and 0 < got[-1] <= 3 * (2048 * d * 4 + 256), (d, got)
        assert L.ffn_norm_workspace_bytes(most + 1, d) == 0 if most < MOST else True
