"""The norms' C ABI on the CPU: sizes, refusals (nothing is launched: every call here fails a check), and the
64-bit reference's gradients against differences."""
import ctypes
import math

import pytest
import torch

from paper_2609_31975_amd import ffn
from tests import norm_ref as ref

L = None
A = 1 << 20                     # a 16-byte-aligned address that is never dereferenced
MIS = A + 4
BIG = 1 << 40


def setup_module(_):
    global L
    L = ffn.lib()


def _form(alpha=1.0, eps=1e-5, post=0, gate_sigmoid=0, gate_rows=0, gate=None, post_gain=None, pre_gain=None):
    return ctypes.byref(ffn.NormStruct(alpha, eps, post, gate_sigmoid, gate_rows, gate, post_gain, pre_gain))


def _fwd(dt=1, T=4, d=64, x=A, f=A, form="plain", x_out=A, n_out=A, rstd=None):
    return L.ffn_norm_forward(dt, T, d, x, f, _form() if form == "plain" else form, x_out, n_out, rstd, None)


def _bwd(dt=1, T=4, d=64, x_out=A, f=A, form="plain", rstd=A, dn=A, dx_out=A, dx=A, df=None, dgate=None, dpost=None,
         dpre=None, ws=A, ws_bytes=BIG):
    return L.ffn_norm_backward(dt, T, d, x_out, f, _form() if form == "plain" else form, rstd, dn, dx_out, dx, df, dgate,
                               dpost, dpre, ws, ws_bytes, None)


@pytest.mark.parametrize("call", [_fwd, _bwd])
def test_shared_refusals(call):
    for dt in (2, 3, 7, -1):
        assert call(dt=dt) == -3
    for kw in ({"T": 0}, {"T": -1}, {"d": 0}, {"d": 16385}, {"T": 1 << 17, "d": 1 << 14}):
        assert call(**kw) == -2, kw
    assert call(form=None) == -1
    for name in ("f", "x_out", "rstd"):
        assert call(**{name: A + 2}) == -4, name
    nan, inf = math.nan, math.inf
    for bad in (dict(eps=0.0), dict(eps=-1e-5), dict(eps=nan), dict(eps=inf), dict(alpha=nan), dict(alpha=inf),
                dict(post=2), dict(post=-1), dict(gate_sigmoid=2, gate=A, gate_rows=1), dict(gate_sigmoid=1),
                dict(gate=A), dict(gate_rows=1), dict(gate=A, gate_rows=2), dict(gate=A, gate_rows=-1),
                dict(post_gain=A)):
        assert call(form=_form(**bad)) == -7, bad
    for bad in (dict(gate=MIS, gate_rows=1), dict(post=1, post_gain=MIS), dict(pre_gain=MIS)):
        assert call(form=_form(**bad)) == -4, bad


def test_forward_refusals():
    assert _fwd(x=None) == -1 and _fwd(x_out=None, n_out=None) == -1
    assert _fwd(x=MIS) == -4 and _fwd(n_out=MIS) == -4
    assert _fwd(n_out=None, form=_form(pre_gain=A)) == -7
    # without a block's output: the norm of x alone
    assert _fwd(f=None) == -7
    for bad in (dict(alpha=0.5), dict(post=1), dict(gate=A, gate_rows=1)):
        assert _fwd(f=None, x_out=None, form=_form(**bad)) == -7, bad


def test_backward_refusals():
    assert _bwd(ws=None) == -1 and _bwd(dn=None, dx_out=None) == -1 and _bwd(dx=None) == -1
    assert _bwd(rstd=None) == -1 and _bwd(x_out=None) == -1
    assert _bwd(rstd=None, dn=None, form=_form(post=1)) == -1
    for name in ("dn", "dx_out", "dx", "df", "dgate", "dpost", "dpre", "ws"):
        assert _bwd(**{name: MIS}) == -4, name
    assert _bwd(f=None, df=A) == -7 and _bwd(dgate=A) == -7 and _bwd(dpost=A) == -7
    assert _bwd(dn=None, dpre=A) == -7
    assert _bwd(ws_bytes=L.ffn_norm_workspace_bytes(4, 64) - 1) == -5


def test_sizes():
    for T, d in ((1, 1), (7, 100), (8192, 8192), (100000, 16384)):
        assert 0 < L.ffn_norm_workspace_bytes(1, d) <= L.ffn_norm_workspace_bytes(T, d) < 1 << 28
    # fewer tokens fit
    sizes = [L.ffn_norm_workspace_bytes(T, 333) for T in (1, 2, 3, 4, 5, 63, 64, 1000, 2047, 2048, 2049, 10 ** 6)]
    assert sizes == sorted(sizes)
    for T, d in ((0, 64), (4, 0), (4, 16385), (1 << 20, 1 << 14)):
        assert L.ffn_norm_workspace_bytes(T, d) == 0


def test_binding_refuses():
    x = torch.zeros(4, 8)
    with pytest.raises(ValueError):
        ffn.ffn_norm_forward(x, x, ffn.norm(1e-5), x, x)       # not on a device
    with pytest.raises(ValueError):
        ffn.norm(1e-5, gate=torch.zeros(8))
    with pytest.raises(ValueError):
        ffn.norm(1e-5, pre_gain=torch.zeros(8))


@pytest.mark.parametrize("post", [False, True])
@pytest.mark.parametrize("gate", [None, "row", "token"])
@pytest.mark.parametrize("sigmoid", [False, True])
def test_reference_gradients(post, gate, sigmoid):
    """backward's formulas against central differences."""
    gen = torch.Generator().manual_seed(1)
    rnd = lambda *s: torch.randn(*s, generator=gen, dtype=torch.float64)
    T, d = 3, 7
    v = {"x": rnd(T, d), "f": rnd(T, d), "pre_gain": rnd(d)}
    if post:
        v["post_gain"] = rnd(d)
    if gate:
        v["gate"] = rnd(1 if gate == "row" else T, d)
    dn, dxo = rnd(T, d), rnd(T, d)

    def form(v):
        return ref.Form(pre_gain=v["pre_gain"], post=post, post_gain=v.get("post_gain"), gate=v.get("gate"), sigmoid=sigmoid,
                        alpha=0.5)

    def loss(v):
        o = ref.forward(v["x"], v["f"], form(v))
        return float((o["n_out"] * dn).sum() + (o["x_out"] * dxo).sum())

    o = ref.forward(v["x"], v["f"], form(v))
    got, _ = ref.backward(o["x_out"], v["f"], form(v), o["rf"], o["r"], dn, dxo, 1)
    for name, value in v.items():
        grad = got["d" + name]
        assert grad.shape == value.shape
        for i in range(value.numel()):
            h = 1e-6
            w = [dict(v, **{name: value + s * h * torch.eye(value.numel(), dtype=torch.float64)[i].view_as(value)}) for s in (1, -1)]
            num = (loss(w[0]) - loss(w[1])) / (2 * h)
            assert abs(num - float(grad.flatten()[i])) < 1e-7 * (1 + abs(num)), (name, i)
