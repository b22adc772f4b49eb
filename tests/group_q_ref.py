"""Products with 4-bit weights and group scales in 64 bits (plain torch on any device), and bounds.

Bounds are elementwise.  U = 2^-24 is half a step of an fp32 value, HALF half a step of the output's type.  A
result is an fp32 sum of (24 + code) x - 24 x, both scaled, and of offset x: K = 3 n_in terms, 9 n_in where fp32 x
is taken apart into three.  Each addition is off by at most U of the partial sum; the errors are independent, and
partial sums are of the size of S, the root of the sum of the terms' squares, so their sum has a deviation of at most
U S sqrt(K / 3), and (8 + 3 sqrt(K)) U S is more than five deviations.  Roundings of the scaled groups are among them.
Through the activation: |A'| and |U'| are at most 1.1 (SiLU's largest slope is 1.0998), and its own arithmetic is
good to 16 U.
"""
import math

import torch

U = 2.0 ** -24
HALF = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}


def codes_of(b):
    c = torch.stack((b & 15, b >> 4), dim=2).reshape(b.shape[0], -1).to(torch.int64)
    return ((c + 8) % 16 - 8).double()


def product(x, codes, scales, offsets):
    """x W^T and the bound of its fp32 sum."""
    c, x = codes_of(codes), x.double()
    g = c.shape[1] // scales.shape[1]
    s = scales.double().repeat_interleave(g, dim=1)
    o = torch.zeros_like(s) if offsets is None else offsets.double().repeat_interleave(g, dim=1)
    w = s * c + o
    size = torch.sqrt((x * x) @ (s * s * ((24 + c) ** 2 + 24 ** 2) + o * o).t())
    return x @ w.t(), (8 + 3 * math.sqrt(9 * c.shape[1])) * U * size


def gated(kind, silu, t, h, eh, v, ev):
    g = h - float(torch.tensor(t, dtype=torch.float32))
    eh = eh + U * (h.abs() + g.abs())
    a = torch.clamp(g, min=0) if kind == 0 else g * torch.sigmoid(g)
    if kind == 1:
        a = torch.where(g > 0, a, torch.zeros_like(a))
    u = v * torch.sigmoid(v) if silu else v
    z = a * u
    return z, 1.1 * eh * u.abs() + 1.1 * ev * a.abs() + 1.21 * eh * ev + 16 * U * z.abs()


def check(got, want, err, dtype, what=""):
    assert got.dtype == dtype and got.shape == want.shape, f"{what}: {got.dtype} {tuple(got.shape)}"
    assert bool(torch.isfinite(got).all()), f"{what}: not finite"
    lim = HALF[dtype] * want.abs() + (1 + HALF[dtype]) * err
    over = (got.double() - want).abs() - lim
    k = int(over.argmax())
    assert float(over.max()) <= 0, (f"{what}: element {k} is {float(got.flatten()[k]):.9g}, want {float(want.flatten()[k]):.9g}, "
                                    f"bound {float(lim.flatten()[k]):.3g}")
