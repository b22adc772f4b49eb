"""Inf and NaN in one request's adapters: they reach the outputs of that request's tokens as the formulas say, through
the projection whose factor holds them and no other, and no other request's token."""
import math

import pytest
import torch

from paper_2609_31975_amd import ffn
from tests import gated_ref as ref

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32
BAD = 2  # the adapter that holds the value

# (dtype, T, d, d_ff, r): the hidden layer in tiles of 16 x 64, cut along k or not, 64 x 64, 128 x 256 and 64 x 128;
# ranks of whole chunks and not
CASES = [(BF16, 12, 136, 200, 8), (F32, 8, 4096, 512, 16), (BF16, 60, 136, 200, 16), (F32, 60, 67, 130, 5),
         (BF16, 130, 72, 100, 9), (BF16, 2100, 136, 2100, 8), (BF16, 2100, 136, 2100, 11), (F32, 600, 264, 1000, 8)]


def positive(gen, shape, std, dtype):
    """Normal values' magnitudes, and no zeros: sums of them and an Inf are that Inf, never NaN."""
    return (torch.randn(shape, generator=gen, device="cuda").abs().clamp_min(2.0 ** -6) * std).to(dtype)


@pytest.mark.parametrize("dtype,T,d,d_ff,r", CASES, ids=lambda v: str(v).replace("torch.", ""))
def test_a_value_in_one_projection_of_the_block(dtype, T, d, d_ff, r):
    """All weights, tokens and factors are positive, so a token of the adapter that holds the value has, in
    64 bits, an output that is all zeros, all Inf of one sign, or all NaN: zeros for a gate of NaN or -Inf, which is
    not above the threshold and beside which the up side is finite; Inf where an Inf is multiplied by what is
    positive."""
    gen = torch.Generator(device="cuda").manual_seed(T + d + r)
    n = 4
    x = positive(gen, (T, d), 1.0, dtype)
    w = [positive(gen, (d_ff, d), d ** -0.5, dtype), positive(gen, (d_ff, d), d ** -0.5, dtype),
         positive(gen, (d_ff, d), d_ff ** -0.5, dtype)]
    pairs = {k: (positive(gen, (n, r, i), i ** -0.5, dtype), positive(gen, (n, o, r), 0.2 * r ** -0.5, dtype))
             for k, (i, o) in {"gate": (d, d_ff), "up": (d, d_ff), "down": (d_ff, d)}.items()}
    ids = torch.randint(-1, n, (T,), generator=gen, device="cuda", dtype=torch.int32)
    ids[:3] = torch.tensor([BAD, 0, BAD], dtype=torch.int32)  # at least two tokens, and another's between them
    own = ids == BAD
    ws = ffn.alloc_gated_workspace(T, d, d_ff, dtype, r, backward=False)
    for kind in (ref.RELU, ref.RSPLUS):
        for name in ("gate", "up"):
            for value in (math.nan, math.inf, -math.inf):
                a = pairs[name][0].clone()
                a[BAD, r - 1, d // 2] = value
                for others in ((name,), ("gate", "up", "down")):
                    some = {k: (a, pairs[k][1]) if k == name else pairs[k] for k in others}
                    y = torch.full_like(x, 7.0)
                    ws.fill_(0xFF)
                    ffn.ffn_gated_forward(x, *w, 0.0, ffn.options(act=kind), y, ws, adapters=ffn.adapters(ids, **some))
                    want = ref.forward(x, *w, 0.0, kind, False, dict(some, ids=ids))["y"]
                    what = f"{name} {value} act {kind} with {'+'.join(others)}"
                    assert not bool((torch.isfinite(want[own]) & (want[own] != 0)).any()), what
                    marks = [torch.nan_to_num(v[own].double(), nan=1.0, posinf=2.0, neginf=-2.0) for v in (y, want)]
                    assert torch.equal(*marks), f"{what}: {y[own][0, :4].tolist()}, not {want[own][0, :4].tolist()}"
                    ref.check(y[~own], want[~own], dtype, 4 if dtype == BF16 else 10, d + d_ff + 2 * r, what)


@pytest.mark.parametrize("dtype,T,d,d_ff,r", CASES, ids=lambda v: str(v).replace("torch.", ""))
def test_a_value_beside_one_neuron(dtype, T, d, d_ff, r):
    """The value in one row of a second factor: with the gate's at NaN or -Inf that neuron alone is off, with any
    other the output of the request's tokens is that Inf or NaN."""
    gen = torch.Generator(device="cuda").manual_seed(T + d + r + 1)
    n = 4
    x = positive(gen, (T, d), 1.0, dtype)
    w = [positive(gen, (d_ff, d), d ** -0.5, dtype), positive(gen, (d_ff, d), d ** -0.5, dtype),
         positive(gen, (d_ff, d), d_ff ** -0.5, dtype)]
    pairs = {k: (positive(gen, (n, r, d), d ** -0.5, dtype), positive(gen, (n, d_ff, r), 0.2 * r ** -0.5, dtype))
             for k in ("gate", "up")}
    ids = torch.randint(-1, n, (T,), generator=gen, device="cuda", dtype=torch.int32)
    ids[:3] = torch.tensor([BAD, 0, BAD], dtype=torch.int32)
    ws = ffn.alloc_gated_workspace(T, d, d_ff, dtype, r, backward=False)
    for name in ("gate", "up"):
        for value in (math.nan, math.inf, -math.inf):
            b = pairs[name][1].clone()
            b[BAD, d_ff // 3, 0] = value
            some = dict(pairs, **{name: (pairs[name][0], b)})
            y = torch.full_like(x, 7.0)
            ws.fill_(0xFF)
            ffn.ffn_gated_forward(x, *w, 0.0, ffn.options(act=ref.RELU), y, ws, adapters=ffn.adapters(ids, **some))
            want = ref.forward(x, *w, 0.0, ref.RELU, False, dict(some, ids=ids))["y"]
            off = name == "gate" and value != math.inf
            own = ids == BAD
            assert bool(torch.isfinite(want[~own]).all()) and bool(torch.isfinite(want[own]).all()) == off
            if not off:
                marks = [torch.nan_to_num(v[own].double(), nan=1.0, posinf=2.0, neginf=-2.0) for v in (y, want)]
                assert torch.equal(*marks), f"{name} {value}: {y[own][0, :4].tolist()}, not {want[own][0, :4].tolist()}"
            rows = slice(None) if off else ~own
            ref.check(y[rows], want[rows], dtype, 4 if dtype == BF16 else 10, d + d_ff + 2 * r, f"{name} {value}")
