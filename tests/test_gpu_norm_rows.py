"""The norms over the most rows that a call takes."""
import math

import pytest
import torch

from paper_2609_31975_amd import ffn
from tests import norm_ref as ref
from tests.test_gpu_norm import BF16, F32, Layer

pytestmark = pytest.mark.gpu


def test_the_most_rows():
    """2^31 - 1 rows of one element that repeat every 2^20: forward and backward, every period as the first, which is held
    to 64 bits."""
    T, few = (1 << 31) - 1, 1 << 20
    layer = Layer(BF16, few, 1)
    n, dx = (torch.full_like(layer.x, math.nan) for _ in range(2))
    rstd = torch.full((2, few), math.nan, dtype=F32, device="cuda")
    form = ffn.norm(1e-5)
    ffn.ffn_norm_forward(layer.x, None, form, None, n, rstd)
    want = ref.forward(layer.x, None, layer.ref)
    ref.check(n, want["n_out"], want["e_n_out"], BF16, "n")
    ffn.ffn_norm_backward(layer.x, None, form, rstd, layer.dn, layer.dxo, ffn.alloc_norm_workspace(few, 1), dx=dx)
    grads, err = ref.backward(layer.x, None, layer.ref, None, rstd[1].double()[:, None], layer.dn, layer.dxo, 1)
    ref.check(dx, grads["dx"], err["dx"], BF16, "dx")

    wide = lambda v: v.repeat(T // few + 1, 1)[:T]
    x, dn, dxo = (wide(v) for v in (layer.x, layer.dn, layer.dxo))
    n_all, rstd_all = torch.full_like(x, math.nan), torch.full((2, T), math.nan, dtype=F32, device="cuda")
    ws = ffn.alloc_norm_workspace(T, 1)
    assert ws.numel() < 1 << 16
    ffn.ffn_norm_forward(x, None, form, None, n_all, rstd_all)
    ffn.ffn_norm_backward(x, None, form, rstd_all, dn, dxo, ws, dx=dxo)
    for got, one, name in ((n_all, n, "n"), (dxo, dx, "dx"), (rstd_all[1], rstd[1], "r")):
        got, one = got.flatten(), one.flatten()
        for a in range(0, T, few * 64):
            part = got[a:a + few * 64]
            assert torch.equal(part, one.repeat(64)[:part.numel()]), (name, a)
