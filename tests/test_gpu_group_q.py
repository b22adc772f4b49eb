"""Products with 4-bit weights and group scales on the GPU against 64 bits (bounds: group_q_ref)."""
import math

import pytest
import torch

from paper_2609_31975_amd import ffn
from tests import group_q_cases
from tests import group_q_ref as ref

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32


class Case:
    def __init__(self, xdt, T, n_in, n_out, group, sdt=F32, offsets=False, seed=0, mats=1):
        gen = torch.Generator(device="cuda").manual_seed(seed * 1000 + T + 3 * n_in + 7 * n_out + group)
        rnd = lambda *s: torch.randn(*s, generator=gen, device="cuda")
        self.xdt, self.T, self.n_in, self.n_out = xdt, T, n_in, n_out
        self.x = rnd(T, n_in).to(xdt)
        self.w, self.q = [], []
        for _ in range(mats):
            codes = torch.randint(0, 256, (n_out, n_in // 2), generator=gen, device="cuda").to(torch.uint8)
            scales = (rnd(n_out, n_in // group) * 0.2 * n_in ** -0.5).to(sdt)
            off = (rnd(n_out, n_in // group) * n_in ** -0.5).to(sdt) if offsets else None
            self.w.append((codes, scales, off))
            self.q.append(ffn.group_q(codes, scales, off))

    def ws(self, gated=False):
        return torch.full_like(ffn.alloc_group_q_workspace(self.T, self.n_in, self.n_out, gated), 0xFF)

    def run(self, ws=None, y=None, **kw):
        y = torch.full((self.T, self.n_out), math.nan, dtype=self.xdt, device="cuda") if y is None else y
        return ffn.ffn_group_q_forward(self.x, self.q[0], y, self.ws() if ws is None else ws, **kw)

    def run_gated(self, t, kind, silu, ws=None, y=None):
        y = torch.full((self.T, self.n_out), math.nan, dtype=self.xdt, device="cuda") if y is None else y
        return ffn.ffn_group_q_gated_forward(self.x, *self.q, t, ffn.options(act=kind, silu_up=silu), y,
                                             self.ws(True) if ws is None else ws)

    def check(self, y, what=""):
        ref.check(y, *ref.product(self.x, *self.w[0]), self.xdt, what)

    def check_gated(self, z, t, kind, silu, what=""):
        h, v = (ref.product(self.x, *w) for w in self.w)
        ref.check(z, *ref.gated(kind, silu, t, *h, *v), self.xdt, what)


# one group; rows behind a tile; a window that ends early; each border of tokens and of x in LDS
TOKENS = [1, 2, 3, 8, 9, 15, 16, 17, 32, 33, 48, 64, 65, 130]


@pytest.mark.parametrize("xdt", [BF16, F32])
@pytest.mark.parametrize("T", TOKENS)
def test_tokens(xdt, T):
    for n_in, group in ((1280, 32), (2304, 128)):
        c = Case(xdt, T, n_in, 333, group, offsets=True)
        c.check(c.run(), f"T={T} group={group}")


@pytest.mark.parametrize("xdt", [BF16, F32])
@pytest.mark.parametrize("n_in,group", [(32, 32), (64, 32), (64, 64), (96, 96), (128, 128), (160, 32), (192, 64), (256, 256), (480, 96),
                                        (640, 160), (768, 384), (1152, 1152), (4096, 4096), (4128, 32), (9216, 128), (28672, 64)])
def test_groups_and_widths(xdt, n_in, group):
    for T, n_out in ((1, 17), (5, 64), (20, 100)):
        c = Case(xdt, T, n_in, n_out, group, sdt=BF16 if T == 5 else F32, offsets=T != 5)
        c.check(c.run(), f"T={T}")


@pytest.mark.parametrize("xdt", [BF16, F32])
@pytest.mark.parametrize("sdt", [BF16, F32])
@pytest.mark.parametrize("offsets", [False, True])
@pytest.mark.parametrize("group", [32, 128])
def test_types(xdt, sdt, offsets, group):
    for T in (1, 7, 24, 50):
        c = Case(xdt, T, 1024, 200, group, sdt, offsets, mats=2)
        c.check(c.run(), f"T={T}")
        c.check_gated(c.run_gated(0.1, 2, False), 0.1, 2, False, f"gated T={T}")


@pytest.mark.parametrize("xdt", [BF16, F32])
@pytest.mark.parametrize("kind", [0, 1, 2])
@pytest.mark.parametrize("silu", [False, True])
def test_gated_forms(xdt, kind, silu):
    for T, n_in, n_out, group in ((1, 512, 1111, 64), (12, 1536, 96, 128), (40, 256, 130, 32)):
        c = Case(xdt, T, n_in, n_out, group, BF16, T == 12, mats=2)
        c.check_gated(c.run_gated(0.25, kind, silu), 0.25, kind, silu, f"T={T}")


@pytest.mark.parametrize("n_out", [1, 15, 16, 64, 4096, 20000])
@pytest.mark.parametrize("T", [1, 33, 64])
def test_rows(n_out, T):
    c = Case(BF16, T, 1024, n_out, 128)
    c.check(c.run())


@pytest.mark.parametrize("xdt", [BF16, F32])
def test_every_code_is_exact(xdt):
    """One x of 1 at a time: the row of weights itself, exactly (the 24 and their removal are whole numbers)."""
    c = Case(xdt, 64, 128, 256, 32, F32)
    c.x.zero_()
    c.x[torch.arange(64), torch.arange(64) * 2] = 1
    y = c.run()
    codes, scales, _ = c.w[0]
    w = (ref.codes_of(codes) * scales.double().repeat_interleave(32, dim=1))[:, ::2].t()
    assert torch.equal(y, w.to(F32).to(xdt))


def test_fp32_tokens_keep_their_bits():
    """One x a token, of 24 bits: six products of it (three parts with 24 + code, three with -24), each sum off by at most
    U of 32 x: 6 * 32 U x.  Without its third part (up to 2^-18 of it, 64 U) a code of 8 would be off by up to 512 U x."""
    c = Case(F32, 64, 128, 256, 32, F32)
    c.w[0][1].fill_(1.0)
    diag = torch.randn(64, device="cuda")
    c.x.zero_()
    c.x[torch.arange(64), torch.arange(64) * 2] = diag
    want = (ref.codes_of(c.w[0][0])[:, ::2] * diag.double()).t()
    assert float(((c.run().double() - want).abs() / diag.double().abs()[:, None]).max()) <= 6 * 32 * ref.U


@pytest.mark.parametrize("bad", [math.inf, math.nan])
def test_special_values(bad):
    for xdt in (BF16, F32):
        c = Case(xdt, 20, 512, 100, 64)
        clean = c.run()
        c.x[7, 100] = bad
        y = c.run()
        keep = torch.arange(20, device="cuda") != 7
        assert torch.equal(y[keep], clean[keep]) and not bool(torch.isfinite(y[7]).any())
        c.x[7, 100] = 0
        c.w[0][1][41, 3] = bad
        clean, y = None, c.run()
        rows = torch.arange(100, device="cuda") != 41
        assert bool(torch.isfinite(y[:, rows]).all()) and not bool(torch.isfinite(y[:, 41]).any())


def test_rows_behind_the_output_stay():
    c = Case(BF16, 3, 256, 50, 64)
    room = torch.full((6, 50), 7.0, dtype=BF16, device="cuda")
    c.run(y=room[:3])
    assert bool((room[3:] == 7).all())


def test_repeats_and_workspaces():
    c, d = Case(BF16, 48, 4096, 640, 128, mats=2), Case(BF16, 2, 4096, 640, 128)
    ws = c.ws(True)
    a = c.run(ws=ws).clone()
    d.check(d.run(ws=ws))       # fewer tokens, the same workspace
    assert torch.equal(a, c.run(ws=ws))
    z = c.run_gated(0.0, 2, False, ws=ws)
    assert torch.equal(z, c.run_gated(0.0, 2, False))


def test_other_stream_and_graphs():
    """On a side stream; two graphs with one workspace, replayed in turn on changing tokens."""
    a, b = Case(BF16, 5, 2048, 512, 128), Case(BF16, 5, 2048, 512, 128, seed=4, mats=2)
    want = a.run(), b.run_gated(0.1, 1, True)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = a.run(stream=side)
    side.synchronize()
    assert torch.equal(got, want[0])
    ws = ffn.alloc_group_q_workspace(5, 2048, 512, gated=True)
    y, z = torch.empty_like(want[0]), torch.empty_like(want[1])
    ga, gb = torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(ga):
        a.run(ws=ws, y=y)
    with torch.cuda.graph(gb):
        b.run_gated(0.1, 1, True, ws=ws, y=z)
    keep = a.x.clone()
    for turn in range(4):
        y.fill_(math.nan), z.fill_(math.nan)
        ga.replay(), gb.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, want[0]) and torch.equal(z, want[1]), turn
        a.x.copy_(b.x)
        ga.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, a.run())
        a.x.copy_(keep)


def test_binding_refusals():
    c = Case(BF16, 4, 128, 64, 64, mats=2)
    y, ws = torch.empty(4, 64, dtype=BF16, device="cuda"), c.ws(True)
    for bad in (dict(x=c.x.float()), dict(x=c.x[:, :64]), dict(x=c.x[0]), dict(y=y.float()), dict(y=y[:3]), dict(ws=ws.cpu())):
        kw = dict(dict(x=c.x, y=y, ws=ws), **bad)
        with pytest.raises((ValueError, TypeError)):
            ffn.ffn_group_q_forward(kw["x"], c.q[0], kw["y"], kw["ws"])
    other = Case(BF16, 4, 128, 32, 64).q[0]
    with pytest.raises(ValueError):
        ffn.ffn_group_q_gated_forward(c.x, c.q[0], other, 0.0, None, y, ws)
    with pytest.raises(ffn.FFNError) as e:
        ffn.ffn_group_q_forward(c.x, c.q[0], y, ws[:16])
    assert e.value.code == -5


@pytest.mark.parametrize("xf32", [0, 1])
@pytest.mark.parametrize("gated", [0, 1])
def test_every_kernel(xf32, gated):
    """The calls that tests/test_group_q_plans.py finds to reach all of them, scales and offsets of either kind in turn."""
    for i, (xf, ga, group, T, n_in, n_out) in enumerate(group_q_cases.CASES):
        if (xf, ga) != (xf32, gated):
            continue
        for sdt, offsets in (((BF16, True), (F32, False)) if i % 2 else ((F32, True), (BF16, False))):
            c = Case(F32 if xf else BF16, T, n_in, n_out, group, sdt, offsets, mats=1 + ga)
            what = f"{group} T={T} {n_in}x{n_out} {sdt} {offsets}"
            if ga:
                c.check_gated(c.run_gated(0.1, 1, True), 0.1, 1, True, what)
            else:
                c.check(c.run(), what)


def test_two_calls_at_once():
    """Two streams with workspaces of their own; more tokens than a pass takes."""
    cases = [Case(F32, T, 1024, 300, 64, BF16, True) for T in (40, 130)]
    want = [c.run().clone() for c in cases]
    streams = [torch.cuda.Stream() for _ in cases]
    torch.cuda.synchronize()
    for _ in range(4):
        outs = []
        for c, st in zip(cases, streams):
            with torch.cuda.stream(st):
                outs.append(c.run())
        torch.cuda.synchronize()
        assert all(torch.equal(o, w) for o, w in zip(outs, want))
