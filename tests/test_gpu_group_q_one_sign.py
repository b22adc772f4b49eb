"""Products with group scales of tokens of one sign, whose sums do not cancel: what the codes' offset of 24 adds to a group's
sum is then many times the result.

Bound, in U = 2^-24: a group's sum is K = 9 group additions at most ((24 + code) x and -24 x, in three parts each, and the
table's), each off by U of a partial sum that is at most A = 31 sum |x| over the group; 8 + 3 sqrt(K) of them are more than five
deviations of their sum (group_q_ref).  Groups are independent: the root of the sum of (scale A)^2.  The scaled groups and
offsets are added in chains of at most G = 3 groups + 64 additions, waves and shares included, of partial sums of at most
the sum of the terms' sizes."""
import math

import pytest
import torch

from paper_2609_31975_amd import ffn
from tests import group_q_ref as ref
from tests.test_gpu_group_q import BF16, F32, Case

pytestmark = pytest.mark.gpu


def bound(x, codes, scales, offsets):
    c, x = ref.codes_of(codes), x.double()
    groups = scales.shape[1]
    g = c.shape[1] // groups
    s = scales.double()
    o = torch.zeros_like(s) if offsets is None else offsets.double()
    a = 31 * x.abs().view(-1, groups, g).sum(2)                                   # [T][groups]
    w = s.repeat_interleave(g, dim=1) * c + o.repeat_interleave(g, dim=1)
    size = x.abs() @ w.abs().t() + x.abs() @ o.abs().repeat_interleave(g, dim=1).t()
    inner = (8 + 3 * math.sqrt(9 * g)) * torch.sqrt((a * a) @ (s * s + o * o).t())
    return x @ w.t(), ref.U * (inner + (3 * groups + 64) * size)


@pytest.mark.parametrize("xdt", [BF16, F32])
@pytest.mark.parametrize("T", [1, 3, 16, 40, 64])
@pytest.mark.parametrize("n_in,group", [(1280, 32), (2304, 128), (1152, 96), (4096, 4096)])
def test_tokens_of_one_sign(xdt, T, n_in, group):
    for offsets in (False, True):
        c = Case(xdt, T, n_in, 333, group, offsets=offsets, mats=2)
        c.x = (c.x.abs() + 0.5).to(xdt)
        h = bound(c.x, *c.w[0])
        ref.check(c.run(), *h, xdt, f"offsets={offsets}")
        ref.check(c.run_gated(0.1, 2, False), *ref.gated(2, False, 0.1, *h, *bound(c.x, *c.w[1])), xdt, f"gated offsets={offsets}")


@pytest.mark.parametrize("sign", ["one", "both"])
@pytest.mark.parametrize("T", [1, 2, 3, 16, 17, 40, 64])
@pytest.mark.parametrize("n_in,group", [(4096, 128), (2048, 64), (1280, 32), (1152, 96)])
def test_fp32_tokens_as_a_sum_of_fp32(sign, T, n_in, group):
    """The norm of the error against that of the result, in U: a group's 3 g additions (three parts of x) are off by U of a
    partial sum each, independently, a deviation of U / sqrt(3) of it at most; codes do not depend on x, so partial sums
    grow in the mean square up to the group's own: sqrt(3 g / 3) of that.  The groups' additions in the same way: sqrt(G).
    Two more for the scales' product and the last rounding.  (Sums that hold 24 times the x beside the codes are 50 U off.)"""
    c = Case(F32, T, n_in, 2048, group)
    if sign == "one":
        c.x = c.x.abs() + 0.5
    want, _ = ref.product(c.x, *c.w[0])
    off = float((c.run().double() - want).norm() / want.norm())
    assert off <= (math.sqrt(group) + math.sqrt(n_in // group) + 2) * ref.U, off / ref.U
