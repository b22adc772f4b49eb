"""The norms around a block, their gradients, and bounds on the kernels' outputs, in 64 bits (plain torch on
any device).

Bounds are elementwise.  U = 2^-24 is half a step of an fp32 value, HALF half a step of the output's type; each
output is rounded once to its type.  A sum over a row adds at most 16 values a thread, then 6 steps of a wave and up to
16 waves: a chain of 38 additions, so it is off by at most 38 U times the sum of its terms' sizes; with the
terms' own products and the division by d, SUM = 44.  r = 1 / sqrt(mean + eps) has half the mean's relative
error (its terms are positive) and the rounding of three operations: 24 U at most.  c = sigma(g): exp to 2 steps, a
sum and a quotient: 6 U.  A product of a few such factors: FACTOR = 40 U of its size.
"""
import torch

HALF = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}
U = 2.0 ** -24
SUM, FACTOR = 44 * U, 40 * U


def mean(v):
    return v.mean(1, keepdim=True)


class Form:
    def __init__(self, eps=1e-5, pre_gain=None, post=False, post_gain=None, gate=None, sigmoid=False, alpha=1.0, pre=True):
        f32 = lambda v: float(torch.tensor(v, dtype=torch.float32))
        self.eps, self.alpha, self.post, self.sigmoid, self.pre = f32(eps), f32(alpha), post, sigmoid, pre
        self.gate, self.post_gain, self.pre_gain = (None if v is None else v.double() for v in (gate, post_gain, pre_gain))

    def c(self):
        """The gate's factor and its slope."""
        if self.gate is None:
            return 1.0, 1.0
        c = torch.sigmoid(self.gate) if self.sigmoid else self.gate
        return c, c * (1 - c) if self.sigmoid else torch.ones_like(c)

    def r(self, v):
        return 1 / torch.sqrt(mean(v * v) + self.eps)


def forward(x, f, form):
    """x', n, the two r (post, pre), and bounds without the outputs' own rounding."""
    x = x.double()
    rf = torch.ones_like(x[:, :1])
    if f is None:
        xo, size = x, torch.zeros_like(x)
    else:
        u = f.double()
        if form.post:
            rf = form.r(u)
            u = u * rf
            if form.post_gain is not None:
                u = u * form.post_gain
        u = u * form.c()[0]
        xo, size = form.alpha * x + u, (form.alpha * x).abs() + u.abs()
    r = form.r(xo)
    pg = 1.0 if form.pre_gain is None else form.pre_gain
    n = xo * r * pg
    kappa = size.norm(dim=1, keepdim=True) / xo.norm(dim=1, keepdim=True).clamp(min=1e-300)
    en = FACTOR * size * (r * pg).abs() if torch.is_tensor(pg) else FACTOR * size * r
    return {"x_out": xo, "n_out": n, "rf": rf, "r": r, "e_x_out": FACTOR * size, "e_n_out": en + n.abs() * (FACTOR * kappa + SUM),
            "e_r": r * (FACTOR * kappa + 24 * U), "e_rf": 24 * U * rf}


def backward(xo, f, form, rf, r, dn, dxo, chain):
    """Gradients for x' and the two r as they are handed over, and their bounds without the outputs' own rounding.
    chain: the longest chain of additions of a sum over the tokens."""
    like = dxo if dxo is not None else dn
    g = torch.zeros_like(like, dtype=torch.float64) if dxo is None else dxo.double()
    eg = U * g.abs()
    out, err = {}, {}
    if dn is not None:
        dn, xh = dn.double(), xo.double() * r
        out["dpre_gain"] = (dn * xh).sum(0)
        err["dpre_gain"] = (chain + 4) * U * (dn * xh).abs().sum(0)
        n = dn if form.pre_gain is None else dn * form.pre_gain
        m = mean(n * xh)
        g = g + r * (n - xh * m)
        eg = 4 * eg + U * r * (6 * n.abs() + 8 * (xh * m).abs()) + r * xh.abs() * SUM * mean((n * xh).abs())
    out["dx"], err["dx"] = form.alpha * g, abs(form.alpha) * (eg + U * g.abs())
    if f is None:
        return out, err
    c, slope = form.c()
    c_abs = c.abs() if torch.is_tensor(c) else c
    fh = f.double() * rf
    og = 1.0 if form.post_gain is None else form.post_gain
    u = fh * og
    if form.gate is not None:
        dg = g * u * slope
        e = (u * slope).abs() * eg + FACTOR * dg.abs() + (8 * U * c_abs * (g * u).abs() if form.sigmoid else 0.0)
        if form.gate.shape[0] == 1:
            out["dgate"] = dg.sum(0, keepdim=True)
            err["dgate"] = e.sum(0, keepdim=True) + (chain + 4) * U * dg.abs().sum(0, keepdim=True)
        else:
            out["dgate"], err["dgate"] = dg, e
    du, edu = g * c, c_abs * eg + 8 * U * (g * c).abs()
    if not form.post:
        out["df"], err["df"] = du, edu
        return out, err
    out["dpost_gain"] = (du * fh).sum(0)
    err["dpost_gain"] = (edu * fh.abs()).sum(0) + (chain + 4) * U * (du * fh).abs().sum(0)
    h = du * og
    eh = edu * (og.abs() if torch.is_tensor(og) else 1.0) + U * h.abs()
    m = mean(h * fh)
    em = mean(eh * fh.abs()) + SUM * mean((h * fh).abs())
    out["df"] = rf * (h - fh * m)
    err["df"] = rf * (eh + fh.abs() * em + 8 * U * (h.abs() + (fh * m).abs()))
    return out, err


def check(got, want, err, dtype, what=""):
    assert got.dtype == dtype and got.shape == want.shape, f"{what}: {got.dtype} {tuple(got.shape)}"
    assert bool(torch.isfinite(got).all()), f"{what}: not finite"
    lim = HALF[dtype] * want.abs() + (1 + HALF[dtype]) * err + 1e-38
    over = (got.double() - want).abs() - lim
    k = int(over.argmax())
    assert float(over.max()) <= 0, (f"{what}: element {k} is {float(got.flatten()[k]):.9g}, want {float(want.flatten()[k]):.9g}, "
                                    f"bound {float(lim.flatten()[k]):.3g}")
