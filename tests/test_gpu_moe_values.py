"""What the experts' hidden values lose on their way into the second product."""
import math

import pytest
import torch

from paper_2609_31975_amd import ffn
from tests import moe_ref as ref
from tests.test_gpu_moe import BF16, Layer

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("shape", [(1, 512, 768, 8, 2), (3, 1024, 2048, 16, 4), (16, 2048, 512, 8, 2), (40, 520, 1000, 6, 3), (64, 256, 1024, 4, 2),
                                   (5, 803, 700, 5, 2), (20, 1001, 333, 4, 2), (7, 1716, 640, 5, 3), (200, 256, 320, 8, 2)])
@pytest.mark.parametrize("kind", [0, 2])
def test_bf16_results_are_rounded_once(shape, kind):
    """The norm of the error is that of y's own rounding to bf16: what the other roundings leave, 2^-18 of z and 64 U of fp32
    sums, is below 1e-5 of y's norm, and a rounding about 1.6e-3.  (z rounded to bf16 would make it 1.4 times as much.)"""
    layer = Layer(BF16, *shape)
    y, ids, weights = layer.run(0.25, kind)
    want, _ = ref.experts(layer.x, *layer.w, 0.25, kind, False, ids, weights)
    once = float((want.to(BF16).double() - want).norm())
    assert float((y.double() - want).norm()) <= 1.02 * once + 1e-5 * float(want.norm())


@pytest.mark.parametrize("shape", [(2, 64, 96, 3, 1), (40, 64, 96, 2, 1)])
def test_a_hidden_value_past_the_range_stays_infinite(shape):
    """A(.) U(.) of one neuron and token is infinite, or rounds to it: an infinite y, no NaN, and the other tokens as they were."""
    for big, up in ((1e38, 10.0), (1.4140625 * 2.0 ** 126, 2.828125)):  # z is infinite; fp32 holds it, its rounding to bf16 is
        layer = Layer(BF16, *shape, given=True)
        layer.ids.zero_()
        layer.weights.fill_(1.0)
        for w in layer.w:
            w.abs_()
        layer.x.abs_()
        clean = layer.run(0.0, 0)[0].clone()
        layer.x[1].zero_()
        layer.x[1, 0] = 1.0
        layer.w[0][0, :, 0].zero_()
        layer.w[1][0, :, 0].zero_()
        layer.w[0][0, 5, 0] = big
        layer.w[1][0, 5, 0] = up
        layer.w[2][0, 5] = layer.w[2][0, 5].clamp(min=1e-3)
        keep = [t for t in range(shape[0]) if t != 1]
        layer.x[:, 0] = torch.where(torch.arange(shape[0], device="cuda") == 1, layer.x[:, 0], torch.zeros_like(layer.x[:, 0]))
        y = layer.run(0.0, 0)[0]
        assert bool((y[1] == math.inf).all()), y[1]
        want, err = ref.experts(layer.x[keep], *layer.w, 0.0, 0, False, layer.ids[keep], layer.weights[keep])
        ref.check(y[keep], want, err, BF16)
        assert bool(torch.isfinite(clean).all())
