"""The gated block and the adapters over more tokens than one launch takes: the calls run in pieces of tokens
(tokens_a_launch), and every token's output is what it is in a call of its own."""
import math

import pytest
import torch

from paper_2609_31975_amd import ffn
from tests import gated_ref as ref

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32


@pytest.fixture(autouse=True)
def room():
    torch.cuda.empty_cache()
    yield
    torch.cuda.empty_cache()


def normal(gen, shape, std, dtype):
    return torch.randn(shape, generator=gen, device="cuda").mul_(std).to(dtype)


def around(T, piece, gen):
    """The first and last tokens of every piece, and some between."""
    at = {t for b in range(0, T, piece) for t in (b, b + 1, b - 1, b - 256, b + 255) if 0 <= t < T} | {T - 1, T - 2}
    return torch.cat([torch.tensor(sorted(at), device="cuda"), torch.randint(0, T, (500,), generator=gen, device="cuda")])


@pytest.mark.parametrize("d", [9, 16], ids=["odd_rows", "whole_chunks"])
def test_projection(d):
    """Three pieces of 2^21 tokens or fewer."""
    T, m, n, r = (1 << 22) + 5, 8, 3, 4
    gen = torch.Generator(device="cuda").manual_seed(d)
    x, w = normal(gen, (T, d), 1.0, BF16), normal(gen, (m, d), d ** -0.5, BF16)
    a, b = normal(gen, (n, r, d), d ** -0.5, BF16), normal(gen, (n, m, r), r ** -0.5, BF16)
    ids = torch.randint(-1, n, (T,), generator=gen, device="cuda", dtype=torch.int32)
    y = torch.full((T, m), math.nan, dtype=BF16, device="cuda")
    ws = ffn.alloc_adapter_workspace(T, d, m, r, BF16)
    ffn.ffn_adapter_forward(x, w, ffn.adapters(ids, gate=(a, b)), y, ws)
    want = x.double() @ w.double().t()
    for j in range(n):
        low = (x.double() @ a[j].double().t()) @ b[j].double().t()
        want += torch.where((ids == j)[:, None], low, torch.zeros_like(low))
    ref.check(y, want, BF16, 2, d + r)


def test_block_with_adapters():
    """Two pieces, adapters on all three projections."""
    T, d, d_ff, n, r = (1 << 21) + 300, 12, 20, 3, 4
    gen = torch.Generator(device="cuda").manual_seed(1)
    x = normal(gen, (T, d), 1.0, F32)
    w = [normal(gen, (d_ff, d), d ** -0.5, F32), normal(gen, (d_ff, d), d ** -0.5, F32), normal(gen, (d_ff, d), d_ff ** -0.5, F32)]
    pairs = {k: (normal(gen, (n, r, i), i ** -0.5, F32), normal(gen, (n, o, r), 0.2 * r ** -0.5, F32))
             for k, (i, o) in {"gate": (d, d_ff), "up": (d, d_ff), "down": (d_ff, d)}.items()}
    ids = torch.randint(-1, n, (T,), generator=gen, device="cuda", dtype=torch.int32)
    y, ws = torch.full_like(x, math.nan), ffn.alloc_gated_workspace(T, d, d_ff, F32, r, backward=False)
    ffn.ffn_gated_forward(x, *w, 0.1, ffn.options(act=2), y, ws, adapters=ffn.adapters(ids, **pairs))
    ref.check(y, ref.forward(x, *w, 0.1, 2, False, dict(pairs, ids=ids))["y"], F32, 10, d + d_ff + 2 * r)


def test_block_of_many_hidden_values():
    """Tokens x columns past 2^35: two pieces (35 GB of hidden values)."""
    T, d, d_ff = (1 << 22) + 300, 8, 4160
    piece = (1 << 35) // (2 * d_ff) // 256 * 256
    assert piece < T
    gen = torch.Generator(device="cuda").manual_seed(2)
    x = normal(gen, (T, d), 1.0, BF16)
    w = [normal(gen, (d_ff, d), s, BF16) for s in (0.35, 0.35, 0.015)]
    y, ws = torch.full_like(x, math.nan), ffn.alloc_gated_workspace(T, d, d_ff, BF16, backward=False)
    ffn.ffn_gated_forward(x, *w, 0.25, ffn.options(act=2), y, ws)
    at = around(T, piece, gen)
    ref.check(y[at], ref.forward(x[at], *w, 0.25, 2)["y"], BF16, 2, d + d_ff)
    assert bool(torch.isfinite(y).all())


def test_training_step():
    """2^27 tokens and some: two pieces, whose g, v and z lie one after the other in the save (86 GB)."""
    T, d, d_ff, piece = (1 << 27) + 300, 8, 3, 1 << 27
    gen = torch.Generator(device="cuda").manual_seed(3)
    x, dy = normal(gen, (T, d), 1.0, BF16), normal(gen, (T, d), 1.0, BF16)
    w = [normal(gen, (d_ff, d), s, BF16) for s in (0.35, 0.35, 0.6)]
    ws, save = ffn.alloc_gated_workspace(T, d, d_ff, BF16), ffn.alloc_gated_save(T, d_ff, BF16)
    y, dx = torch.full_like(x, math.nan), torch.full_like(x, math.nan)
    dw = [torch.full_like(v, math.nan) for v in w]
    opt = ffn.options(act=2)
    ffn.ffn_gated_forward(x, *w, 0.25, opt, y, ws, save=save)
    ffn.ffn_gated_backward(x, *w, opt, dy, save, dx, *dw, ws)
    del save, ws
    at = around(T, piece, gen)
    f = ref.forward(x[at], *w, 0.25, 2)
    ref.check(y[at], f["y"], BF16, 2, d + d_ff, "y")
    ref.check(dx[at], ref.backward(x[at], *w, dy[at], f)["dx"], BF16, 2, 2 * (d + d_ff), "dx")
    total = None
    for k in range(0, T, 1 << 22):
        xs, dys = x[k:k + (1 << 22)], dy[k:k + (1 << 22)]
        g = ref.backward(xs, *w, dys, ref.forward(xs, *w, 0.25, 2))
        total = {n: g[n] if total is None else total[n] + g[n] for n in g if n != "dx"}
    for n, got in zip(("dw_gate", "dw_up", "dw_down_t"), dw):
        ref.check(got, total[n], BF16, 2, T + 2 * d, n)
