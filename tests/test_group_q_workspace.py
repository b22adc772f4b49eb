"""The workspace of the products with group scales: room for the shares that a call makes and no more, swept on the CPU
with the library's own plans."""
import random
import shutil

import pytest

from paper_2609_31975_amd import ffn
from tests.test_gated_launches import compile_driver
from tests.test_group_q_plans import plans


def sizes():
    rng = random.Random(11)
    out = []
    for _ in range(20000):
        group = 32 * rng.choice([1, 1, 2, 3, 4, 4, 5, 8])
        n_in = group * max(1, int(2 ** rng.uniform(0, 20) / group))
        n_out = int(2 ** rng.uniform(0, 20))
        if n_in * n_out < 1 << 31:
            out.append((rng.randint(0, 1), rng.randint(0, 1), group, rng.randint(1, 64), n_in, n_out))
    # many shares: few rows of great length, and each side of what fills the card
    for n_out in (1, 15, 16, 17, 1024, 2048, 2049, 4096, 8192, 8193, 16384, 16385):
        for T in (1, 2, 16, 17, 48, 64):
            for xf32 in (0, 1):
                for gated in (0, 1):
                    out.append((xf32, gated, 128, T, 1 << 16, n_out))
    return out


def rest(T, n_in):
    """Bytes of x in parts and of the table of its sums, in whole 256 bytes each: as many columns as a workgroup's two waves
    take at once, whole tiles of 16 tokens."""
    columns = -(-n_in // 256) * 256
    up = lambda n: -(-n // 256) * 256
    return up(6 * (-(-min(T, 64) // 16) * 16) * columns) + up(4 * columns // 32 * 64)


@pytest.mark.skipif(shutil.which("g++") is None, reason="needs g++")
def test_shares_fit_and_little_is_left(tmp_path):
    L = ffn.lib()
    cases = sizes()
    shared = 0
    for c, p in zip(cases, plans(compile_driver("group_q_plans_driver", tmp_path), cases)):
        _, gated, _, T, n_in, n_out = c
        room = L.ffn_group_q_workspace_bytes(T, n_in, n_out, gated) - rest(T, n_in)
        if p["shares"] > 1:
            shared += 1
            assert room >= 4 * p["shares"] * (1 + gated) * T * n_out, (c, p, room)
        # 512 workgroups of 32 rows of weights or 256 of 64, at the very most
        assert 0 <= room <= 4 * (1 + gated) * T * 16384 + 256, (c, p, room)
    assert shared > 1000


def test_a_large_head_needs_little():
    L = ffn.lib()
    # 64 tokens through a head of 128256 rows: x in parts, 3 MB, and nothing beside it
    assert L.ffn_group_q_workspace_bytes(64, 8192, 128256, 0) == rest(64, 8192)
    assert L.ffn_group_q_workspace_bytes(64, 64, 1 << 20, 1) == rest(64, 64)
    for gated in (0, 1):
        for n_in, n_out in ((4096, 100), (4096, 8192), (8192, 8193), (64, 1 << 20), (1 << 20, 64)):
            got = [L.ffn_group_q_workspace_bytes(T, n_in, n_out, gated) for T in (1, 2, 15, 16, 17, 33, 63, 64, 65, 1000)]
            assert got == sorted(got) and got[0] > 0
