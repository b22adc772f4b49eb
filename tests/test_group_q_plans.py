"""The tiles of the products with group scales: the library's own host arithmetic, swept on the CPU by a small driver
linked to it."""
import random
import shutil
import subprocess

import pytest

from tests import group_q_cases
from tests.test_gated_launches import compile_driver

pytestmark = pytest.mark.skipif(shutil.which("g++") is None, reason="needs g++")

NAMES = "nt wk u whole ns chunk per_share shares blocks lds".split()


def plans(exe, cases):
    text = "".join(" ".join(map(str, c)) + "\n" for c in cases)
    res = subprocess.run([exe], input=text, capture_output=True, text=True, check=True)
    out = [dict(zip(NAMES, map(int, line.split()))) for line in res.stdout.splitlines()]
    assert len(out) == len(cases)
    return out


@pytest.fixture(scope="module")
def exe(tmp_path_factory):
    return compile_driver("group_q_plans_driver", tmp_path_factory.mktemp("plans"))


def test_every_plan_fits(exe):
    rng = random.Random(3)
    cases = []
    for _ in range(60000):
        group = 32 * rng.choice([1, 1, 2, 2, 3, 4, 4, 5, 8, 12, 40])
        n_in = group * max(1, int(2 ** rng.uniform(0, 20) / group))
        n_out = int(2 ** rng.uniform(0, 20))
        if n_in * n_out < 1 << 31:
            cases.append((rng.randint(0, 1), rng.randint(0, 1), group, rng.randint(1, 64), n_in, n_out))
    for c, p in zip(cases, plans(exe, cases)):
        xf32, gated, group, T, n_in, n_out = c
        unit, windows = p["wk"] * p["u"], -(-n_in // (128 if p["nt"] else 256))
        assert p["nt"] == (0 if T == 1 else -(-T // 16)), c
        assert p["chunk"] >= unit and p["chunk"] % unit == 0 and p["per_share"] % unit == 0, (c, p)
        assert 1 <= p["shares"] <= 8 and (p["shares"] - 1) * p["per_share"] < windows <= p["shares"] * p["per_share"], (c, p)
        assert p["lds"] <= (64 if p["nt"] <= 1 else 160) * 1024, (c, p)
        assert p["blocks"] * (8 // p["wk"] * 16) >= n_out and p["blocks"] * p["shares"] < 1 << 22, (c, p)
        assert p["ns"] == (1 if group % 128 == 0 else 8 if n_in % 128 else {64: 2, 32: 4}.get(group, 8)), (c, p)
        batch = 1 if gated or p["ns"] > 1 else 2
        if p["nt"] == 0:
            assert p["u"] == 1 and p["wk"] in (2, 4, 8), (c, p)
        elif p["nt"] == 1 and p["whole"]:
            assert p["u"] == batch and p["wk"] in (2, 4, 8) and p["chunk"] == p["per_share"], (c, p)
        elif p["nt"] == 1:
            # the pieces of x that a thread holds
            assert p["u"] == 1 and p["wk"] in ((4, 8) if xf32 else (8,)) and T * p["chunk"] * 16 <= 512 * (2 if xf32 else 4), (c, p)
        else:
            assert p["u"] == 1 and p["wk"] == 2 and p["chunk"] == 2, (c, p)


def test_the_cases_reach_every_kernel(exe):
    reached, shared = set(), set()
    for c, p in zip(group_q_cases.CASES, plans(exe, group_q_cases.CASES)):
        kind = (p["wk"],) if p["nt"] == 0 else (p["wk"], p["whole"], p["ns"]) if p["nt"] == 1 else (p["ns"],)
        reached.add((c[0], c[1], p["nt"], *kind))
        if p["shares"] > 1:
            shared.add((c[0], c[1], min(p["nt"], 2)))
    want = set()
    for xf32 in (0, 1):
        for gated in (0, 1):
            want |= {(xf32, gated, 0, wk) for wk in (2, 4, 8)}
            want |= {(xf32, gated, 1, wk, 1, ns) for wk in (2, 4, 8) for ns in (1, 2, 4, 8)}
            want |= {(xf32, gated, 1, wk, 0, ns) for wk in ((4, 8) if xf32 else (8,)) for ns in (1, 2, 4, 8)}
            want |= {(xf32, gated, nt, ns) for nt in (2, 3, 4) for ns in (1, 2, 4, 8)}
    assert want <= reached, sorted(want - reached)
    assert shared == {(x, g, t) for x in (0, 1) for g in (0, 1) for t in (0, 1, 2)}, shared
