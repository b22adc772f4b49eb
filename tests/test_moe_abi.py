"""The mixture-of-experts layer's C ABI on the CPU: sizes and refusals (nothing is launched: every call here
fails a check)."""
import ctypes
import math

import pytest
import torch

from paper_2609_31975_amd import ffn
from tests import moe_ref as ref

L = None
A = 1 << 20                     # a 16-byte-aligned address that is never dereferenced
MIS = A + 4
BIG = 1 << 50


def setup_module(_):
    global L
    L = ffn.lib()


def _r(experts=8, k=2, w=A, bias=None, sigmoid=0, normalize=0, scale=1.0):
    return ctypes.byref(ffn.RouterStruct(experts, k, w, bias, sigmoid, normalize, scale))


def _fwd(wdt=1, T=4, d=64, d_ff=96, r="plain", x=A, g=A, u=A, dn=A, opt=None, ids=A, weights=A, y=A, ws=A, ws_bytes=BIG):
    return L.ffn_moe_forward(wdt, T, d, d_ff, _r() if r == "plain" else r, x, g, u, dn, ctypes.c_float(0.5), opt, ids, weights,
                             y, ws, ws_bytes, None)


def test_refusals():
    for name in ("r", "x", "g", "u", "dn", "ids", "weights", "y", "ws"):
        assert _fwd(**{name: None}) == -1, name
    for name in ("x", "g", "u", "dn", "y", "ws"):
        assert _fwd(**{name: MIS}) == -4, name
    assert _fwd(ids=A + 2) == -4 and _fwd(weights=A + 1) == -4
    for wdt in (2, 3, -1):
        assert _fwd(wdt=wdt) == -3
    for kw in ({"T": 0}, {"T": 257}, {"d": 0}, {"d_ff": 0}, {"d": (1 << 20) + 8}, {"d_ff": (1 << 20) + 1},
               {"d": 1 << 16, "d_ff": 1 << 15}, {"T": 256, "d_ff": 1 << 20, "d": 8}):
        assert _fwd(**kw) == -2, kw
    for kw in (dict(experts=0), dict(experts=513), dict(k=0), dict(k=9), dict(k=17, experts=64), dict(experts=-1)):
        assert _fwd(r=_r(**kw)) == -2, kw
    for kw in (dict(w=MIS), dict(bias=A + 2)):
        assert _fwd(r=_r(**kw)) == -4, kw
    for kw in (dict(sigmoid=2), dict(normalize=-1), dict(scale=math.inf), dict(scale=math.nan)):
        assert _fwd(r=_r(**kw)) == -7, kw
    # a given routing has no router's fields
    for kw in (dict(bias=A, scale=0.0), dict(sigmoid=1, scale=0.0), dict(normalize=1, scale=0.0), dict(scale=1.0)):
        assert _fwd(r=_r(w=None, **kw)) == -7, kw
    for opt in (dict(act=3), dict(silu_up=2), dict(rms_norm=1, rms_eps=1e-6), dict(g_idx=A, g_sign=A)):
        assert _fwd(opt=ctypes.byref(ffn.Options(**opt))) == -7, opt
    need = L.ffn_moe_workspace_bytes(1, 4, 64, 96, 8, 2)
    assert need > 0 and _fwd(ws_bytes=need - 1) == -5


def test_sizes():
    sizes = [L.ffn_moe_workspace_bytes(1, T, 512, 1000, 64, 6) for T in (1, 2, 15, 16, 17, 64, 255, 256)]
    assert sizes == sorted(sizes)
    for bad in ((2, 4, 64, 96, 8, 2), (1, 0, 64, 96, 8, 2), (1, 257, 64, 96, 8, 2), (1, 4, 64, 96, 8, 9), (1, 4, 64, 96, 600, 2)):
        assert L.ffn_moe_workspace_bytes(*bad) == 0


def test_binding_refuses():
    with pytest.raises(ValueError):
        ffn.router(8, 2, w=torch.zeros(7, 64))
    with pytest.raises(ValueError):
        ffn.router(8, 2, bias=torch.zeros(8))
    with pytest.raises(ValueError):
        ffn.router(8, 2, w=torch.zeros(8, 64))     # not on a device


def test_reference():
    """The routing and the layer of the reference by hand."""
    x = torch.tensor([[1.0, 0.0], [0.0, 2.0]])
    w = torch.tensor([[1.0, 0.0], [0.0, 1.0], [1.0, 0.0]])
    ids, s = ref.route(x, w, None, 2, False, True, 1.0)
    assert ids.tolist() == [[0, 2], [1, 0]] and abs(float(s[0, 0]) - 0.5) < 1e-12
    assert abs(float(s[1, 0]) - 1 / (1 + math.exp(-2))) < 1e-12
    ids, s = ref.route(x, w, torch.tensor([0.0, 5.0, 0.1]), 1, True, False, 2.0)
    assert ids.tolist() == [[1], [1]] and abs(float(s[0, 0]) - 1.0) < 1e-12
    wg, wu, wd = torch.ones(3, 1, 2), torch.ones(3, 1, 2), torch.ones(3, 1, 2)
    y, _ = ref.experts(x, wg, wu, wd, 0.0, 0, False, torch.tensor([[0, -1], [2, 2]]), torch.tensor([[0.5, 9.0], [1.0, 0.25]]))
    assert y.tolist() == [[0.5, 0.5], [5.0, 5.0]]
