"""The norms' forward calls that keep nothing for a backward call (rstd None), whose rows are read past the caches, and calls of
more rows than workgroups: against 64 bits (bounds: norm_ref) and, bit by bit, against the calls that keep rstd."""
import math

import pytest
import torch

from paper_2609_31975_amd import ffn
from tests import norm_ref as ref
from tests.test_gpu_norm import BF16, F32, KINDS, SIZES, Layer

pytestmark = pytest.mark.gpu


def forward(layer, x_out=True, n_out=True, rstd=False, x=None):
    x = layer.x if x is None else x
    o = {n: torch.full_like(x, math.nan) if on else None for n, on in (("x_out", x_out), ("n_out", n_out and layer.pre))}
    o["rstd"] = torch.full((2, layer.T), math.nan, dtype=F32, device="cuda") if rstd else None
    ffn.ffn_norm_forward(x, layer.f, layer.form, o["x_out"], o["n_out"], o["rstd"])
    return o


def check(layer, o, what=""):
    want = ref.forward(layer.x, layer.f, layer.ref)
    for name in ("x_out", "n_out"):
        if o[name] is not None:
            ref.check(o[name], want[name], want["e_" + name], layer.dtype, f"{what} {name}")


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("T,d", SIZES)
def test_sizes(dtype, T, d):
    layer = Layer(dtype, T, d, **KINDS["token"])
    got, kept = forward(layer), forward(layer, rstd=True)
    check(layer, got, f"T={T} d={d}")
    for name in ("x_out", "n_out"):
        assert torch.equal(got[name], kept[name]), name
        alone = forward(layer, **{"n_out" if name == "x_out" else "x_out": False}) if name == "n_out" else None
        assert alone is None or torch.equal(alone["n_out"], got["n_out"])


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("kind", list(KINDS))
@pytest.mark.parametrize("T,d", [(1, 96), (37, 1000), (11, 2500), (5, 6001), (3, 9000)])
def test_forms(dtype, kind, T, d):
    layer = Layer(dtype, T, d, **KINDS[kind])
    got, kept = forward(layer), forward(layer, rstd=True)
    check(layer, got, kind)
    assert all(got[n] is None or torch.equal(got[n], kept[n]) for n in ("x_out", "n_out"))


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("T,d", [(40, 1536), (6, 1001), (9, 2048), (5, 4096), (5, 4099), (4, 8192), (3, 12000), (2, 9001)])
def test_in_place(dtype, T, d):
    """x_out over x itself."""
    layer = Layer(dtype, T, d, **KINDS["token"])
    want = forward(layer)
    x, n = layer.x.clone(), torch.full_like(layer.x, math.nan)
    ffn.ffn_norm_forward(x, layer.f, layer.form, x, n)
    assert torch.equal(x, want["x_out"]) and torch.equal(n, want["n_out"])


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("d", [40, 1001, 1536, 2500, 8192, 16383])
def test_norm_alone(dtype, d):
    """Before a first block."""
    layer = Layer(dtype, 6, d, gains=True)
    n = torch.full_like(layer.x, math.nan)
    ffn.ffn_norm_forward(layer.x, None, layer.form, None, n)
    want = ref.forward(layer.x, None, layer.ref)
    ref.check(n, want["n_out"], want["e_n_out"], dtype)


@pytest.mark.parametrize("bad", [math.inf, math.nan])
def test_special_values_stay_in_their_token(bad):
    for d in (1000, 1001, 2048, 4096, 5001, 9000):
        layer = Layer(BF16, 13, d, **KINDS["row"])
        clean = forward(layer)
        layer.x[4, 17] = bad
        got = forward(layer)
        keep = torch.arange(13, device="cuda") != 4
        for name in ("x_out", "n_out"):
            assert torch.equal(got[name][keep], clean[name][keep]), (d, name)
        assert not bool(torch.isfinite(got["n_out"][4]).all())


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("T,d", [(5, 33), (2, 1032), (3, 1001), (2, 2048), (1, 4095), (2, 4096), (2, 5000), (1, 16383)])
def test_what_lies_behind_the_rows_stays(dtype, T, d):
    layer = Layer(dtype, T, d, **KINDS["token"])
    want = forward(layer)
    rooms = [torch.full((T * d + 4096,), 7.0, dtype=dtype, device="cuda") for _ in range(2)]
    ffn.ffn_norm_forward(layer.x, layer.f, layer.form, *(r[:T * d].view(T, d) for r in rooms))
    for r, name in zip(rooms, ("x_out", "n_out")):
        assert torch.equal(r[:T * d].view(T, d), want[name]) and bool((r[T * d:] == 7).all()), name


@pytest.mark.parametrize("d", [1032, 1025])
def test_more_rows_than_workgroups(d):
    """2^20 workgroups of a row each and some rows more: a workgroup's second row is normed as a first one is.  The rows
    repeat every 96, so the outputs have to."""
    T, few = (1 << 20) + 96, 96
    T -= T % few
    assert T > 1 << 20
    layer = Layer(BF16, few, d, post=True, gains=True, gate="row", sigmoid=True)
    want = forward(layer)
    check(layer, want)
    wide = lambda v: v.repeat(T // few, 1)
    x, f = wide(layer.x), wide(layer.f)
    n_out = torch.full_like(x, math.nan)
    ffn.ffn_norm_forward(x, f, layer.form, x, n_out)
    for got, name in ((x, "x_out"), (n_out, "n_out")):
        # bits compared: NaN never equals itself
        assert bool((got.view(T // few, few, d) == want[name]).all()), name
