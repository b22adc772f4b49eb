"""Every path of the calls with adapters (adapter_cases) against 64 bits, and one request's Inf and NaN kept from the
others on each of them (bounds: gated_ref)."""
import math

import pytest
import torch

from paper_2609_31975_amd import ffn
from tests import gated_ref as ref
from tests.adapter_cases import CASES

pytestmark = pytest.mark.gpu

BAD = 2  # the adapter that comes to hold an Inf or NaN


def normal(gen, shape, std, dtype):
    return (torch.randn(shape, generator=gen, device="cuda") * std).to(dtype)


class Call:
    def __init__(self, op, f32, T, d, n, r):
        gen = torch.Generator(device="cuda").manual_seed(T + 3 * d + 5 * n + 7 * r + f32)
        self.block, self.T, self.d, self.n, self.r = op == "b", T, d, n, r
        self.dtype = torch.float32 if f32 else torch.bfloat16
        count = 7
        self.x = normal(gen, (T, d), 1.0, self.dtype)
        sizes = {"gate": (d, n), "up": (d, n), "down": (n, d)} if self.block else {"gate": (d, n)}
        self.w = [normal(gen, (n, d), (n if name == "down" else d) ** -0.5, self.dtype) for name in sizes]
        size = 0.2 if self.block else 1.0
        self.pairs = {name: (normal(gen, (count, r, i), i ** -0.5, self.dtype),
                             normal(gen, (count, o, r), size * r ** -0.5, self.dtype)) for name, (i, o) in sizes.items()}
        self.scale = 0.5 + torch.rand(count, generator=gen, device="cuda")
        self.ids = torch.randint(-1, count, (T,), generator=gen, device="cuda", dtype=torch.int32)
        # another request's token first, and tokens of BAD beside it; a token without an adapter last
        first = torch.tensor([0, BAD, 5, BAD][:T], dtype=torch.int32)
        self.ids[:len(first)] = first
        if T > 5:
            self.ids[-1] = -1

    def run(self, pairs):
        ad = ffn.adapters(self.ids, scale=self.scale, **pairs)
        if not self.block:
            y = torch.full((self.T, self.n), math.nan, dtype=self.dtype, device="cuda")
            ws = torch.full_like(ffn.alloc_adapter_workspace(self.T, self.d, self.n, self.r, self.dtype), 0xFF)
            return ffn.ffn_adapter_forward(self.x, self.w[0], ad, y, ws)
        y = torch.full_like(self.x, math.nan)
        ws = torch.full_like(ffn.alloc_gated_workspace(self.T, self.d, self.n, self.dtype, self.r, backward=False), 0xFF)
        return ffn.ffn_gated_forward(self.x, *self.w, 0.1, ffn.options(act=2, silu_up=True), y, ws, adapters=ad)

    def want(self):
        if self.block:
            return ref.forward(self.x, *self.w, 0.1, 2, True, dict(self.pairs, ids=self.ids, scale=self.scale))["y"]
        return self.x.double() @ self.w[0].double().t() + ref.low_rank(self.x.double(), self.ids, *self.pairs["gate"], self.scale)

    def check(self, got, want, what):
        bf16 = self.dtype == torch.bfloat16
        if self.block:  # z, A x on its way into g and v, A z, and the output
            ref.check(got, want, self.dtype, 4 if bf16 else 10, self.d + self.n + 2 * self.r, what)
        else:  # A x, and the output
            ref.check(got, want, self.dtype, 2 if bf16 else 4, self.d + self.r, what)


@pytest.mark.parametrize("case", CASES, ids=lambda c: "-".join(map(str, c)))
def test_path(case):
    call = Call(*case)
    clean, want = call.run(call.pairs), call.want()
    call.check(clean, want, "clean")
    assert torch.equal(call.run(call.pairs), clean)
    own = call.ids == BAD
    for name, (a, b) in call.pairs.items():
        for value in (math.nan, math.inf):
            for which in (0, 1):
                bad = [a.clone(), b.clone()]
                bad[which][BAD, bad[which].shape[1] // 2, bad[which].shape[2] - 1] = value
                got = call.run(dict(call.pairs, **{name: tuple(bad)}))
                what = f"{value} in {name}'s {'ab'[which]}"
                call.check(got[~own], want[~own], what)
                if bool(own.any()):
                    assert not bool(torch.isfinite(got[own]).all(dim=1).any()), what
                else:
                    assert torch.equal(got, clean), what
