"""The experts' launches and workspace: the library's own host arithmetic, swept on the CPU by a small driver linked to it."""
import random
import shutil
import subprocess

import pytest

from paper_2609_31975_amd import ffn
from tests.test_gated_launches import compile_driver


def valid(f32, T, d, d_ff, E, k):
    return k <= E and d * d_ff < 1 << 31 and T * k * (-(-d_ff // 32) * 32) < 1 << 29


def sizes():
    rng = random.Random(5)
    out = []
    while len(out) < 30000:
        E = int(2 ** rng.uniform(0, 9.001))
        c = (rng.randint(0, 1), int(2 ** rng.uniform(0, 8.001)), int(2 ** rng.uniform(0, 20)), int(2 ** rng.uniform(0, 20)), E,
             rng.randint(1, min(E, 16)))
        if valid(*c):
            out.append(c)
    return out


@pytest.mark.skipif(shutil.which("g++") is None, reason="needs g++")
def test_every_plan_fits_its_workspace(tmp_path):
    L = ffn.lib()
    cases = sizes()
    text = "".join(" ".join(map(str, c)) + "\n" for c in cases)
    res = subprocess.run([compile_driver("moe_plans_driver", tmp_path)], input=text, capture_output=True, text=True, check=True)
    lines = [tuple(map(int, line.split())) for line in res.stdout.splitlines()]
    assert len(lines) == len(cases)
    up = lambda n: -(-n // 256) * 256
    cut = 0
    for c, p in zip(cases, lines):
        f32, T, d, d_ff, E, k = c
        slots, ldz, pieces, rows = p
        assert slots == min(T * k, E) and ldz % 32 == 0 and 0 <= ldz - d_ff < 32, (c, p)
        columns = -(-d // (64 if f32 else 128))
        # four waves of a workgroup take 32 neurons each of a piece
        assert 1 <= pieces <= 8 and (pieces == 1 or pieces * 128 <= ldz), (c, p)
        assert slots <= 512 and columns * 256 < 1 << 32 and ldz // 16 * 256 < 1 << 32, (c, p)  # HIP's limits, grid dimension by dimension
        # what the pieces leave fits, and little room is left: at most as many rows as workgroups fill the card, or a row a place
        assert pieces * T * k <= rows <= 8 * T * k and rows <= T * k + (-(-1024 // columns) - 1) * -(-T * k // E), (c, p)
        assert L.ffn_moe_workspace_bytes(0 if f32 else 1, T, d, d_ff, E, k) == \
            up(8 * T * E) + up(4 * T * k * ldz) + up(4 * rows * d), (c, p)
        cut += pieces > 1
    assert cut > 3000


def test_a_large_layer_needs_little():
    """256 tokens, 8 of 64 experts of 7168: the neurons are in one piece, whose rows are 59 MB; sizes grow with the tokens."""
    L = ffn.lib()
    assert L.ffn_moe_workspace_bytes(1, 256, 7168, 2048, 64, 8) < 80e6
    for wdt, d, d_ff, E, k in ((1, 7168, 2048, 64, 8), (0, 4096, 14336, 8, 2), (1, 64, 10000, 16, 1), (1, 100, 33, 3, 3), (0, 1, 1 << 18, 512, 16),
                               (1, 128, 1 << 14, 512, 3)):
        got = [L.ffn_moe_workspace_bytes(wdt, T, d, d_ff, E, k) for T in range(1, 65)]
        assert got == sorted(got) and got[0] > 0
