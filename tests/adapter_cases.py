"""Sizes of calls with adapters that reach every path they can take, the smallest that do; test_adapter_plans.py
holds them to that, test_gpu_adapter_paths.py runs them.

A path is a tile (with its last tiles cut along k or not, and rows of the rank whole 16-byte chunks or not) of the hidden
layer's, the down or the projection call's product, or a kind of A x: through LDS tiles or not, rows of whole chunks or not,
in shares or not, for one stack or the block's two."""
import itertools
import subprocess

# ("b" the block with adapters on all three projections, "p" the projection call; fp32; T, d, d_ff or n_out, r)
CASES = [
    ("b", 0, 1, 64, 64, 5), ("b", 1, 1, 64, 64, 5), ("b", 0, 1, 137, 65, 8), ("b", 1, 1, 137, 65, 8),
    ("b", 0, 2100, 64, 64, 5), ("b", 1, 2100, 64, 64, 5), ("b", 1, 1, 2048, 2100, 5), ("b", 1, 1, 2050, 2101, 8),
    ("b", 0, 24, 4096, 64, 8), ("b", 0, 24, 64, 4100, 8), ("b", 0, 65, 64, 5000, 5), ("b", 1, 1100, 520, 64, 8),
    ("b", 1, 2100, 64, 1000, 5), ("b", 0, 1100, 4096, 64, 5), ("b", 0, 65, 64, 64, 8), ("b", 1, 24, 520, 512, 8),
    ("b", 0, 1, 1032, 1000, 5), ("b", 0, 1, 1032, 1000, 8), ("b", 1, 1100, 1032, 64, 5), ("b", 1, 2100, 2048, 64, 8),
    ("b", 1, 130, 1032, 4100, 8), ("b", 1, 65, 2050, 4100, 5), ("b", 0, 4200, 2048, 1000, 5), ("b", 0, 4200, 2048, 1000, 8),
    ("p", 0, 2100, 1032, 64, 5), ("p", 0, 1, 64, 64, 5), ("p", 0, 1, 64, 64, 8), ("p", 1, 1, 64, 64, 5),
    ("p", 1, 1, 64, 64, 8), ("p", 0, 24, 64, 64, 8), ("p", 1, 24, 64, 64, 5), ("p", 1, 24, 64, 64, 8),
    ("p", 0, 65, 64, 64, 5), ("p", 0, 65, 64, 64, 8), ("p", 1, 1, 520, 64, 5), ("p", 1, 1, 520, 64, 8),
    ("p", 1, 24, 520, 64, 5), ("p", 1, 24, 520, 64, 8), ("p", 0, 1, 1032, 64, 5), ("p", 0, 1, 1032, 64, 8),
    ("p", 0, 24, 1032, 64, 5), ("p", 0, 24, 1032, 64, 8), ("p", 1, 4200, 64, 200, 5), ("p", 1, 4200, 64, 200, 8),
    ("p", 1, 2100, 2048, 65, 5), ("p", 1, 2100, 2048, 65, 8), ("p", 0, 4200, 4096, 200, 5), ("p", 0, 4200, 4096, 200, 8),
    # several adapters in the tiles of a few tokens, and ranks of more than one workgroup's 16 or 64
    ("b", 0, 12, 4096, 512, 24), ("b", 1, 15, 2048, 264, 20), ("b", 0, 60, 2048, 520, 40), ("b", 0, 1100, 2048, 2100, 72),
    ("b", 0, 2100, 2048, 2100, 64), ("p", 1, 6, 4096, 500, 36), ("p", 0, 3000, 4096, 1000, 128), ("p", 1, 2100, 1032, 100, 68)]

# what is swept for the paths that there are
SWEEP = list(itertools.product(
    "bp", (0, 1), (1, 6, 12, 16, 24, 40, 60, 64, 65, 80, 130, 200, 300, 400, 600, 1100, 1500, 2100, 3000, 4200),
    (64, 136, 137, 264, 520, 1032, 1033, 2048, 2050, 4096), (64, 65, 200, 512, 1000, 1001, 2100, 2101, 4100, 5000), (5, 8)))


def paths(exe, cases):
    """The paths of each case, from the driver adapter_paths_driver.cpp."""
    text = "\n".join(" ".join(map(str, c)) for c in cases)
    out = subprocess.run([exe], input=text, capture_output=True, text=True, check=True).stdout.splitlines()
    assert len(out) == len(cases)
    found = []
    for (_, f32, _, d, n, r), line in zip(cases, out):
        whole = 4 if f32 else 8
        keys = set()
        for words in (part.split() for part in line.split(";") if part):
            k = {"x": d, "z": n}.get(words[0], r)
            name = "A x" if words[0] in "xz" else words[0]
            keys.add((f32, name, *words[1:], k % whole == 0))
        found.append(keys)
    return found
