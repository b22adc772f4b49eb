"""A mixture-of-experts layer in 64 bits (plain torch on any device), and bounds.

Bounds are elementwise.  U = 2^-24 is half a step of an fp32 value, HALF half a step of the tokens' type.  An
fp32 sum of K terms whose squares' sum has the root S is off by at most (8 + 3 sqrt(K)) U S (group_q_ref), the
activation's result by what its arguments' errors make of it (the same).  z is rounded to the tokens' type: errors
of at most HALF |z|, independent, with deviations of HALF |z| / sqrt(3) at most: 3 times the root of the sum of
(HALF z w)^2 is over five deviations of their part of a sum.  The errors of z before its rounding are those of
sums of their own, independent as well: their part is the root of the sum of (ez w)^2.  The weighted sum over a token's
experts and the weights' own rounding: 32 U of the sum of its terms' sizes (16 experts at most).  y is rounded once.
"""
import math

import torch

from tests import group_q_ref as q

U, HALF = q.U, q.HALF


def route(x, w, bias, k, sigmoid, normalize, scale):
    """ids, weights; equal scores go to the lower index (a stable sort), a NaN score counts as the lowest."""
    logits = x.double() @ w.double().t()
    score = torch.sigmoid(logits) if sigmoid else torch.softmax(logits, dim=1)
    by = logits if bias is None else score + bias.double()
    ids = torch.sort(by, dim=1, descending=True, stable=True).indices[:, :k]
    s = score.gather(1, ids)
    if normalize:
        s = s / s.sum(1, keepdim=True)
    return ids.to(torch.int32), s * float(torch.tensor(scale, dtype=torch.float32))


def experts(x, wg, wu, wd, t, kind, silu, ids, weights):
    """y and its bound without y's own rounding, for the routing as it is handed over."""
    T, d = x.shape
    E, d_ff, _ = wg.shape
    half = HALF[x.dtype]
    x = x.double()
    y, err, size = (torch.zeros(T, d, dtype=torch.float64, device=x.device) for _ in range(3))
    for e in sorted(set(int(i) for i in ids.flatten().tolist() if 0 <= i < E)):
        tok, place = (ids == e).nonzero(as_tuple=True)
        xe, g, u, w = x[tok], wg[e].double(), wu[e].double(), wd[e].double()
        terms = (8 + 3 * math.sqrt(d)) * U
        eh, ev = (terms * torch.sqrt((xe * xe) @ (m * m).t()) for m in (g, u))
        z, ez = q.gated(kind, silu, t, xe @ g.t(), eh, xe @ u.t(), ev)
        w2 = w * w
        f = z @ w
        ef = 3 * half * torch.sqrt((z * z) @ w2) + torch.sqrt((ez * ez) @ w2) + (8 + 3 * math.sqrt(d_ff)) * U * torch.sqrt((z * z) @ w2)
        s = weights[tok, place].double()[:, None]
        y.index_add_(0, tok, s * f)
        err.index_add_(0, tok, s.abs() * ef)
        size.index_add_(0, tok, (s * f).abs())
    return y, err + 32 * U * size


check = q.check
