"""Values at which the norms' arithmetic is hardest: gates that saturate, rows whose squares pass fp32's range."""
import math

import pytest
import torch

from paper_2609_31975_amd import ffn
from tests import norm_ref as ref
from tests.test_gpu_norm import BF16, F32, Layer

pytestmark = pytest.mark.gpu

U = ref.U


@pytest.mark.parametrize("gate_rows", [1, 2])
def test_the_gate_s_slope_where_it_saturates(gate_rows):
    """dgate = dx_out f sigma (1 - sigma), relative to itself however small 1 - sigma is (no norms: G is dx_out, u is f).

    Roundings, in U = 2^-24: 2^(-g log2 e) 2 (one unit in the last place) and 1 for its rest, so 3 in 1 - sigma's numerator; the
    denominator at most as many and its own, 4; the quotient's reciprocal and Newton step 2; so sigma 6, 1 - sigma (numerator
    times it) 3 + 6 + 1, their product 17, f dx_out 1, the last product 1: 19.  Products below 2^-126 are rounded to a multiple of 2^-149, by
    half of that.  One row: a sum of one token, exact."""
    d = 4096
    gen = torch.Generator(device="cuda").manual_seed(5)
    T = gate_rows
    gate = torch.linspace(-80, 80, T * d, device="cuda").view(T, d)
    f, dxo = (torch.randn((T, d), generator=gen, device="cuda") for _ in range(2))
    form = ffn.norm(1e-5, gate=gate, gate_sigmoid=True)
    dgate = torch.full_like(gate, math.nan)
    ffn.ffn_norm_backward(None, f, form, None, None, dxo, ffn.alloc_norm_workspace(T, d), dgate=dgate)
    g = gate.double()
    want = dxo.double() * f.double() * torch.sigmoid(g) * torch.sigmoid(-g)
    over = (dgate.double() - want).abs() - (20 * U * want.abs() + 2.0 ** -150)
    k = int(over.argmax())
    assert float(over.max()) <= 0, (float(g.flatten()[k]), float(dgate.flatten()[k]), float(want.flatten()[k]))


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("d", [64, 512, 1000, 1001, 1536, 4096, 5001, 8192, 9000, 16384])
def test_rows_whose_squares_pass_the_range(dtype, d):
    """Finite rows of up to a tenth of the largest number are normed as any other, in the block's output and in the
    residual, beside ordinary rows and rows with an infinity."""
    layer = Layer(dtype, 9, d, post=True, gains=True, gate="row", sigmoid=True)
    row = torch.randn(d, generator=torch.Generator(device="cuda").manual_seed(d), device="cuda").clamp(-3, 3)
    big = lambda s: (row * s).to(dtype)
    layer.x[1], layer.x[2], layer.x[3] = big(1e20), big(3e25), big(1e37)
    layer.f[4], layer.f[5], layer.f[6] = big(1e19), big(1e37), big(5e30)
    layer.x[6] = big(2e30)
    clean = layer.run()
    layer.check(clean, what=f"d={d}")
    n, x_out = torch.full_like(layer.x, math.nan), torch.full_like(layer.x, math.nan)
    ffn.ffn_norm_forward(layer.x, layer.f, layer.form, x_out, n)
    assert torch.equal(n, clean["n_out"]) and torch.equal(x_out, clean["x_out"])
    layer.x[7, d // 2], layer.f[8, 0] = math.inf, math.inf
    got = layer.run()
    for name in ("x_out", "n_out", "dx", "df"):
        assert torch.equal(got[name][:7], clean[name][:7]), name
        assert name == "dx" or not bool(torch.isfinite(got["n_out"][7:]).all(dim=1).any())
