"""The gated block's and the adapters' C ABI on the CPU: sizes, refusals (nothing is launched: every call
here fails a check), and the 64-bit reference's gradients against differences."""
import ctypes

import pytest
import torch

from paper_2609_31975_amd import ffn
from tests import gated_ref as ref

L = None
A = 1 << 20                     # a 16-byte-aligned address that is never dereferenced
MIS = A + 4
BIG = 1 << 40


def setup_module(_):
    global L
    L = ffn.lib()


def _ad(n=4, r=8, ids=A, scale=None, **kw):
    return ctypes.byref(ffn.AdapterStruct(n, r, ids, scale, *(kw.get(k) for k in ("gate_a", "gate_b", "up_a", "up_b",
                                                                                  "down_a", "down_b"))))


def _opt(**kw):
    return ctypes.byref(ffn.Options(**kw))


def _fwd(wdt=1, T=4, d=64, d_ff=128, x=A, g=A, u=A, dn=A, opt=None, ad=None, y=A, save=None, save_bytes=0, ws=A,
         ws_bytes=BIG):
    return L.ffn_gated_forward(wdt, T, d, d_ff, x, g, u, dn, ctypes.c_float(0.5), opt, ad, y, save, save_bytes, ws,
                               ws_bytes, None)


def _bwd(wdt=1, T=4, d=64, d_ff=128, x=A, g=A, u=A, dn=A, opt=None, dy=A, save=A, save_bytes=BIG, dx=A, dg=A, du=A,
         dd=A, ws=A, ws_bytes=BIG):
    return L.ffn_gated_backward(wdt, T, d, d_ff, x, g, u, dn, opt, dy, save, save_bytes, dx, dg, du, dd, ws, ws_bytes,
                                None)


def _adp(wdt=1, T=4, d=64, n=128, x=A, w=A, ad="gate", y=A, ws=A, ws_bytes=BIG):
    ad = _ad(gate_a=A, gate_b=A) if ad == "gate" else ad
    return L.ffn_adapter_forward(wdt, T, d, n, x, w, ad, y, ws, ws_bytes, None)


@pytest.mark.parametrize("call", [_fwd, _bwd, _adp])
def test_shared_refusals(call):
    assert call(x=None) == -1 and call(ws=None) == -1
    for wdt in (2, 3, 7, -1):
        assert call(wdt=wdt) == -3
    size = "n" if call is _adp else "d_ff"
    for kw in ({"T": 0}, {"d": 0}, {"d": -8}, {size: 0}, {"d": (1 << 20) + 8}, {size: (1 << 20) + 1},
               {"d": 1 << 16, size: 1 << 15}, {"T": 1 << 30, "d": 64}):
        assert call(**kw) == -2, kw
    assert call(x=MIS) == -4 and call(ws=MIS) == -4


def test_forward_refusals():
    for name in ("g", "u", "dn", "y"):
        assert _fwd(**{name: None}) == -1 and _fwd(**{name: MIS}) == -4
    need = ffn.lib().ffn_gated_workspace_bytes(1, 4, 64, 128, 0, 0)
    assert _fwd(ws_bytes=need - 1) == -5
    save = ffn.lib().ffn_gated_save_bytes(1, 4, 128)
    assert _fwd(save=A, save_bytes=save - 1) == -5 and _fwd(save=MIS, save_bytes=save) == -4
    for opt in (dict(act=3), dict(act=-1), dict(silu_up=2), dict(rms_norm=1, rms_eps=1e-6), dict(g_idx=A, g_sign=A),
                dict(rms_gain=A)):
        assert _fwd(opt=_opt(**opt)) == -7, opt
    # every activation passes the checks up to the workspace's
    for a in range(3):
        assert _fwd(opt=_opt(act=a, silu_up=1), ws_bytes=need - 1) == -5


def test_backward_refusals():
    for name in ("g", "u", "dn", "dy", "save"):
        assert _bwd(**{name: None}) == -1 and _bwd(**{name: MIS}) == -4
    assert _bwd(dx=None, dg=None, du=None, dd=None) == -1
    for name in ("dx", "dg", "du", "dd"):
        assert _bwd(**{name: MIS}) == -4
    assert _bwd(save_bytes=ffn.lib().ffn_gated_save_bytes(1, 4, 128) - 1) == -5
    # the forward call's workspace is not enough for the backward call's
    assert _bwd(ws_bytes=ffn.lib().ffn_gated_workspace_bytes(1, 4, 64, 128, 0, 0)) == -5
    assert _bwd(opt=_opt(act=5)) == -7


def test_adapter_refusals():
    pair = dict(gate_a=A, gate_b=A)
    for call in (lambda **k: _fwd(ad=_ad(**k)), lambda **k: _adp(ad=_ad(**k))):
        assert call() == -1                                   # no projection has any
        assert call(ids=None, **pair) == -1
        assert call(gate_a=A) == -1 and call(gate_b=A) == -1  # half a pair
        assert call(n=0, **pair) == -2 and call(r=0, **pair) == -2 and call(r=1 << 17, **pair) == -2
        assert call(gate_a=MIS, gate_b=A) == -4 and call(gate_a=A, gate_b=MIS) == -4
        assert call(ids=A + 2, **pair) == -4 and call(scale=A + 1, **pair) == -4
    assert _fwd(ad=_ad(up_a=A, **pair)) == -1
    assert _adp(ad=_ad(up_a=A, up_b=A, **pair)) == -7 and _adp(ad=_ad(down_a=A, down_b=A)) == -1
    assert _adp(ad=None) == -1
    save = ffn.lib().ffn_gated_save_bytes(1, 4, 128)
    assert _fwd(ad=_ad(**pair), save=A, save_bytes=save) == -7
    # the workspace grows with the rank
    need = ffn.lib().ffn_gated_workspace_bytes(1, 4, 64, 128, 8, 0)
    assert need > ffn.lib().ffn_gated_workspace_bytes(1, 4, 64, 128, 0, 0)
    assert _fwd(ad=_ad(**pair), ws_bytes=need - 1) == -5
    assert _adp(ws_bytes=ffn.lib().ffn_adapter_workspace_bytes(1, 4, 64, 128, 8) - 1) == -5


def test_the_decode_calls_refuse_the_new_activation():
    rc = L.ffn_sparse_forward_ex(1, 1, 64, 128, A, A, A, A, ctypes.c_float(0.5), _opt(act=ffn.FFN_ACT_SILU), A, A, BIG,
                                 None)
    assert rc == -7


def test_sizes():
    for wdt in (0, 1):
        f = L.ffn_gated_workspace_bytes(wdt, 4096, 4096, 14336, 0, 0)
        b = L.ffn_gated_workspace_bytes(wdt, 4096, 4096, 14336, 0, 1)
        assert 0 < f < b
        assert L.ffn_gated_save_bytes(wdt, 4096, 14336) > 2 * 4 * 4096 * 14336
    for bad in ((2, 4, 64, 128, 0, 0), (1, 0, 64, 128, 0, 0), (1, 4, 0, 128, 0, 0), (1, 4, 64, 128, -1, 0),
                (1, 4, 64, 128, 1 << 17, 0), (1, 4, 1 << 16, 1 << 15, 0, 0)):
        assert L.ffn_gated_workspace_bytes(*bad) == 0, bad
    assert L.ffn_gated_save_bytes(1, 0, 8) == 0 and L.ffn_gated_save_bytes(3, 8, 8) == 0
    assert L.ffn_adapter_workspace_bytes(1, 8, 64, 64, 0) == 0
    with pytest.raises(ffn.FFNError):
        ffn.alloc_gated_save(0, 8, torch.float32, device="cpu")
    with pytest.raises(TypeError):
        ffn.alloc_gated_save(1, 8, torch.float16, device="cpu")


@pytest.mark.parametrize("wdt", [0, 1])
def test_a_workspace_serves_fewer_tokens_and_lower_ranks(wdt):
    tokens = [1, 2, 7, 15, 16, 17, 48, 63, 64, 65, 100, 127, 128, 129, 255, 257, 400, 513, 777, 1000, 2047, 2049, 3000,
              4096, 6000, 12288, 12289, 20000, 60000]
    for d, d_ff in ((64, 128), (1000, 2731), (1001, 2731), (4096, 14336), (8192, 28672)):
        for r in (0, 1, 8, 16, 17, 24, 33, 64, 128):
            low = 0
            for T in tokens:
                for back in (0, 1):
                    n = L.ffn_gated_workspace_bytes(wdt, T, d, d_ff, r, back)
                    assert n >= L.ffn_gated_workspace_bytes(wdt, T, d, d_ff, max(0, r - 1), back) > 0
                assert n >= low
                low = n
            if r:
                sizes = [L.ffn_adapter_workspace_bytes(wdt, T, d, d_ff, r) for T in tokens]
                assert sizes == sorted(sizes) and sizes[0] > 0


def test_binding_refuses_host_tensors():
    x, w = torch.zeros(2, 8), torch.zeros(16, 8)
    with pytest.raises(ValueError):
        ffn.ffn_gated_forward(x, w, w, w, 0.0, None, x, x)
    with pytest.raises(ValueError):
        ffn.adapters(torch.zeros(2, dtype=torch.int32), gate=(torch.zeros(1, 4, 8), torch.zeros(1, 16, 4)))


@pytest.mark.parametrize("kind,silu", [(ref.RELU, False), (ref.RSPLUS, True), (ref.SILU, True)])
def test_reference_gradients_are_differences(kind, silu):
    """Central differences with a step of 1e-5 in 64 bits: 1e-10 of truncation and 1e-11 of rounding on
    values near 1, so 1e-7 of the gradient's norm."""
    gen = torch.Generator().manual_seed(3)
    T, d, d_ff = 5, 7, 11
    x, wg, wu, wd = (torch.randn(*s, generator=gen, dtype=torch.float64) for s in ((T, d), (d_ff, d), (d_ff, d), (d_ff, d)))
    dy = torch.randn(T, d, generator=gen, dtype=torch.float64)
    t = ref.threshold_in_gap(x @ wg.t(), 0.3)
    grads = ref.backward(x, wg, wu, wd, dy, ref.forward(x, wg, wu, wd, t, kind, silu))

    def loss(*p):
        return float((ref.forward(*p, t, kind, silu)["y"] * dy).sum())

    for k, name in enumerate(("dx", "dw_gate", "dw_up", "dw_down_t")):
        p = [x, wg, wu, wd]
        dirn = torch.randn(p[k].shape, generator=gen, dtype=torch.float64)
        dirn /= dirn.norm()
        e = 1e-5
        hi, lo = list(p), list(p)
        hi[k], lo[k] = p[k] + e * dirn, p[k] - e * dirn
        diff = (loss(*hi) - loss(*lo)) / (2 * e)
        want = float((grads[name] * dirn).sum())
        assert abs(diff - want) <= 1e-7 * float(grads[name].norm()), name
