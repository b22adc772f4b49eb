"""The gated block, its gradients and adapters in 64 bits (plain torch on any device), and the bounds that
the kernels' outputs are held to.

Bounds.  A rounding to a type is off by at most half a step, HALF of the value.  Where `n` roundings lie
between exact inputs and an output (z or dg or A_j x on its way into a product, and the output's own), every
term of the output carries errors of at most HALF each; those of different terms are independent, so the
output as a whole is off by at most sqrt(n) HALF of its norm.  fp32 sums of K terms: each addition is off by half a
step of the partial sum, a random walk, (4 + sqrt(K)) 2^-24 of the norm with K the terms of the longest chain
of sums (bf16 products are summed in fp32 as well).  Single rows (a token's output, a neuron's gradient)
hold fewer terms: twice that, of their own norm and the mean row's.

g = h - t is a difference.  Its error is that of h's sum and of the subtraction, (4 + sqrt(K)) 2^-24 of s =
sqrt(sum of the squares of the sum's terms, and of t), whatever is left of it: where few neurons pass the
threshold, and by little, that is many times 2^-24 of g.  It enters z as e A'(g) U(v) and dv as dz e A'(g) U'(v),
so beside the terms' own |A(g) U(v)| it weighs f = |s A'(g) U(v)| / |A(g) U(v)| (and without U for dv; the
larger of both, as norms over the whole or over the row), and the fp32 part of a bound is 1 + f times as large.
"""
import math

import torch

HALF = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}
RELU, RSPLUS, SILU = 0, 1, 2


def act(kind, g):
    """A(g) and A'(g)."""
    on = (g > 0).to(g.dtype)
    if kind == RELU:
        return torch.where(g > 0, g, torch.zeros_like(g)), on
    s = torch.sigmoid(g)
    a, da = g * s, s * (1 + g * (1 - s))
    if kind == SILU:
        return a, da
    zero = torch.zeros_like(g)
    return torch.where(g > 0, a, zero), torch.where(g > 0, da, zero)


def up(silu, v):
    if not silu:
        return v, torch.ones_like(v)
    s = torch.sigmoid(v)
    return v * s, s * (1 + v * (1 - s))


def low_rank(x, ids, a, b, scale):
    """scale_j B_j (A_j x) per token; zero where the token has no adapter."""
    out = torch.zeros(x.shape[0], b.shape[1], dtype=x.dtype, device=x.device)
    for j in sorted(set(int(i) for i in ids.tolist() if 0 <= i < a.shape[0])):
        rows = (ids == j).nonzero().flatten()
        s = 1.0 if scale is None else scale[j].double()
        out[rows] = s * ((x[rows] @ a[j].double().t()) @ b[j].double().t())
    return out


def forward(x, wg, wu, wd, t, kind=RELU, silu=False, ad=None):
    """ad: dict with ids, scale and pairs by projection."""
    x, wg, wu, wd = (w.double() for w in (x, wg, wu, wd))

    def low(name, z):
        return low_rank(z, ad["ids"], *ad[name], ad.get("scale")) if ad and ad.get(name) else 0.0

    g = x @ wg.t() + low("gate", x) - t
    v = x @ wu.t() + low("up", x)
    a, da = act(kind, g)
    u, du = up(silu, v)
    z = a * u
    return {"y": z @ wd + low("down", z), "g": g, "v": v, "a": a, "da": da, "u": u, "du": du, "z": z}


def backward(x, wg, wu, wd, dy, f):
    x, wg, wu, wd, dy = (w.double() for w in (x, wg, wu, wd, dy))
    dz = dy @ wd.t()
    dg, dv = dz * f["u"] * f["da"], dz * f["a"] * f["du"]
    return {"dx": dg @ wg + dv @ wu, "dw_gate": dg.t() @ x, "dw_up": dv.t() @ x, "dw_down_t": f["z"].t() @ dy}


def threshold_in_gap(h, near):
    """A threshold close to `near` that no gate value comes close to: the middle of the widest gap among
    the values around it (the derivative of a ReLU jumps there, and a sum that rounds to the other side gives
    another right answer)."""
    h = h.double().flatten().sort().values
    at = int(torch.searchsorted(h, torch.tensor(float(near), dtype=h.dtype, device=h.device)))
    lo, hi = max(0, at - 50), min(len(h), at + 50)
    if hi - lo < 2:
        return float(near)
    gaps = h[lo + 1:hi] - h[lo:hi - 1]
    k = int(gaps.argmax())
    t = float(torch.tensor(float((h[lo + k] + h[lo + k + 1]) / 2), dtype=torch.float32))
    assert float((h - t).abs().min()) > 1e-7 * (1 + abs(t)), "no gap around the threshold"
    return t


def difference(x, wg, t, f):
    """f of the docstring above: over all elements, per token and per neuron."""
    s = torch.sqrt((x.double() ** 2) @ (wg.double() ** 2).t() + float(t) ** 2)
    out = []
    for dim in (None, 1, 0):
        best = None
        for u in (f["u"], torch.ones_like(f["u"])):
            over, under = (s * f["da"] * u).norm(dim=dim), (f["a"] * u).norm(dim=dim)
            q = torch.where(under > 0, over / under, torch.zeros_like(over))
            best = q if best is None else torch.maximum(best, q)
        out.append(best)
    return out


def bound(dtype, roundings, terms, f=0.0):
    return math.sqrt(roundings) * HALF[dtype] + (4 + math.sqrt(terms)) * 2.0 ** -24 * (1 + f)


def check(got, ref, dtype, roundings, terms, what="", f=0.0, f_rows=0.0):
    assert got.dtype == dtype and got.shape == ref.shape, f"{what}: {got.dtype} {tuple(got.shape)}"
    b = bound(dtype, roundings, terms, float(f))
    ref = ref.to(got.device)
    err = got.double() - ref
    assert bool(torch.isfinite(got).all()), f"{what}: not finite"
    norm = float(ref.norm())
    if norm == 0:
        assert not bool(got.any()), f"{what}: not zero"
        return
    assert float(err.norm()) <= b * norm, f"{what}: {float(err.norm()) / norm:.3e} of the norm, bound {b:.3e}"
    rows, ref_rows = err.norm(dim=1), ref.norm(dim=1)
    lim = 2 * bound(dtype, roundings, terms, torch.clamp(torch.as_tensor(f_rows), min=float(f))) * (ref_rows + ref_rows.mean())
    bad = (rows > lim).nonzero().flatten()
    assert not len(bad), f"{what}: rows {bad[:8].tolist()} off by {rows[bad[:4]].tolist()}, bounds {lim[bad[:4]].tolist()}"
    dead = ref_rows == 0
    assert not bool(got[dead].any()), f"{what}: rows that are zero are not"
