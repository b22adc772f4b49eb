"""The C ABI of the products with group scales on the CPU: sizes and refusals (nothing is launched: every call
here fails a check)."""
import ctypes

import pytest
import torch

from paper_2609_31975_amd import ffn
from tests import group_q_ref as ref

L = None
A = 1 << 20                     # a 16-byte-aligned address that is never dereferenced
MIS = A + 4
BIG = 1 << 40


def setup_module(_):
    global L
    L = ffn.lib()


def _q(codes=A, scales=A, offsets=None, sdt=1, group=64):
    return ctypes.byref(ffn.GroupQStruct(codes, scales, offsets, sdt, group))


def _one(xdt=1, T=4, n_in=128, n_out=96, x=A, w="plain", y=A, ws=A, ws_bytes=BIG, **_):
    return L.ffn_group_q_forward(xdt, T, n_in, n_out, x, _q() if w == "plain" else w, y, ws, ws_bytes, None)


def _two(xdt=1, T=4, n_in=128, n_out=96, x=A, w="plain", w2="plain", opt=None, y=A, ws=A, ws_bytes=BIG):
    return L.ffn_group_q_gated_forward(xdt, T, n_in, n_out, x, _q() if w == "plain" else w, _q() if w2 == "plain" else w2,
                                       ctypes.c_float(0.5), opt, y, ws, ws_bytes, None)


@pytest.mark.parametrize("call", [_one, _two])
def test_refusals(call):
    for name in ("x", "w", "y", "ws"):
        assert call(**{name: None}) == -1, name
    for name in ("x", "y", "ws"):
        assert call(**{name: MIS}) == -4, name
    for xdt in (2, 3, -1, 9):
        assert call(xdt=xdt) == -3
    for kw in ({"T": 0}, {"n_in": 0}, {"n_out": 0}, {"n_out": -3}, {"n_in": (1 << 20) + 64}, {"n_out": (1 << 20) + 1},
               {"n_in": 1 << 16, "n_out": 1 << 15}, {"T": 1 << 24}):
        assert call(**kw) == -2, kw
    assert call(w=_q(codes=None)) == -1 and call(w=_q(scales=None)) == -1
    for sdt in (2, 3, -1):
        assert call(w=_q(sdt=sdt)) == -3
    for group in (0, -32, 1, 16, 48, 96, 256):
        assert call(w=_q(group=group)) == -2, group
    for kw in (dict(codes=MIS), dict(scales=MIS), dict(offsets=MIS)):
        assert call(w=_q(**kw)) == -4, kw
    need = L.ffn_group_q_workspace_bytes(4, 128, 96, int(call is _two))
    assert need > 0 and call(ws_bytes=need - 1) == -5


def test_gated_refusals():
    assert _two(w2=None) == -1 and _two(w2=_q(codes=None)) == -1
    assert _two(w2=_q(sdt=0)) == -7 and _two(w2=_q(group=32)) == -7 and _two(w2=_q(offsets=A)) == -7
    for opt in (dict(act=3), dict(act=-1), dict(silu_up=2), dict(rms_norm=1, rms_eps=1e-6), dict(g_idx=A, g_sign=A)):
        assert _two(opt=ctypes.byref(ffn.Options(**opt))) == -7, opt


def test_sizes():
    for gated in (0, 1):
        sizes = [L.ffn_group_q_workspace_bytes(T, 4096, 4096, gated) for T in (1, 2, 8, 16, 17, 33, 64, 65, 4096)]
        assert sizes == sorted(sizes) and sizes[0] > 0
    for bad in ((0, 64, 64, 0), (1, 0, 64, 0), (1, 64, 0, 0), (1, 64, 64, 2), (1, 1 << 21, 64, 0)):
        assert L.ffn_group_q_workspace_bytes(*bad) == 0


def test_binding_refuses():
    b, s = torch.zeros(8, 32, dtype=torch.uint8), torch.zeros(8, 2)
    for args in ((b, s), (b.int(), s), (b, s[:4]), (b, torch.zeros(8, 3)), (b, s, s.bfloat16())):
        with pytest.raises((ValueError, TypeError)):
            ffn.group_q(*args)


def test_reference_codes():
    """Nibbles by hand, and unsigned codes with a zero point as the header gives them."""
    b = torch.tensor([[0x70, 0xF8]], dtype=torch.uint8)
    assert ref.codes_of(b).tolist() == [[0.0, 7.0, -8.0, -1.0]]
    u, p, scale = torch.tensor([3, 15, 0, 9]), 5, 0.5
    packed = torch.tensor([[3 | 15 << 4, 0 | 9 << 4]], dtype=torch.uint8) ^ 0x88
    w = ref.codes_of(packed) * scale + scale * (8 - p)
    assert w.tolist() == [(scale * (u - p)).tolist()]
