"""The gated block and its backward pass on the GPU against 64 bits (bounds: gated_ref)."""
import math

import pytest
import torch

from paper_2609_31975_amd import ffn
from tests import gated_ref as ref

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32


class Layer:
    """A layer's weights, tokens and output gradient, values of the scale of a trained one."""

    def __init__(self, dtype, T, d, d_ff, seed=0, near=0.6):
        gen = torch.Generator(device="cuda").manual_seed(seed * 1000 + T + 7 * d + 13 * d_ff)

        def normal(shape, std):
            return (torch.randn(shape, generator=gen, device="cuda") * std).to(dtype)

        self.dtype, self.T, self.d, self.d_ff = dtype, T, d, d_ff
        self.x, self.dy = normal((T, d), 1.0), normal((T, d), 1.0)
        self.w = [normal((d_ff, d), d ** -0.5), normal((d_ff, d), d ** -0.5), normal((d_ff, d), d_ff ** -0.5)]
        self.t = ref.threshold_in_gap(self.x.double() @ self.w[0].double().t(), near)

    def forward(self, kind=0, silu=False, t=None, save=None, ws=None, y=None, x=None, **kw):
        t = self.t if t is None else t
        x = self.x if x is None else x
        if ws is None:
            ws = torch.full_like(ffn.alloc_gated_workspace(x.shape[0], self.d, self.d_ff, self.dtype), 0xFF)
        y = torch.full_like(x, math.nan) if y is None else y
        return ffn.ffn_gated_forward(x, *self.w, t, ffn.options(act=kind, silu_up=silu), y, ws, save=save, **kw)

    def train(self, kind=0, silu=False, t=None, ws=None, want=(True,) * 4, **kw):
        save = torch.full_like(ffn.alloc_gated_save(self.T, self.d_ff, self.dtype), 0xFF)
        if ws is None:
            ws = torch.full_like(ffn.alloc_gated_workspace(self.T, self.d, self.d_ff, self.dtype), 0xFF)
        y = self.forward(kind, silu, t, save, ws, **kw)
        ws.fill_(0xFF)  # the forward call leaves nothing there that the backward call reads
        outs = [torch.full_like(w, math.nan) if on else None for w, on in zip((self.x, *self.w), want)]
        ffn.ffn_gated_backward(self.x, *self.w, ffn.options(act=kind, silu_up=silu), self.dy, save, *outs, ws, **kw)
        return dict(zip(("y", "dx", "dw_gate", "dw_up", "dw_down_t"), (y, *outs)))

    def reference(self, kind=0, silu=False, t=None):
        """Gradients, y, and the factors of gated_ref.difference."""
        f = ref.forward(self.x, *self.w, self.t if t is None else t, kind, silu)
        f["f"] = ref.difference(self.x, self.w[0], self.t if t is None else t, f)
        return dict(ref.backward(self.x, *self.w, self.dy, f), y=f["y"], f=f["f"])

    def check(self, got, kind=0, silu=False, t=None, what=""):
        want = self.reference(kind, silu, t)
        terms = {"y": self.d_ff + self.d, "dx": 2 * self.d_ff + 2 * self.d, "dw_gate": self.T + 2 * self.d,
                 "dw_up": self.T + 2 * self.d, "dw_down_t": self.T + self.d}
        for name, g in got.items():
            if g is not None:
                # z, dg or dv once, and the output; fp32: the same two, and the activation's own arithmetic
                f, tok, neu = want["f"]
                ref.check(g, want[name], self.dtype, 2 if self.dtype == BF16 else 8, terms[name], f"{what} {name}", f,
                          neu if name.startswith("dw") else tok)


# sizes around every tile's edges and steps: rows 16 / 64 / 128 / 256, columns 64 / 128 / 256, k 32 / 64
FORWARD = [(1, 8, 1), (1, 64, 64), (2, 72, 65), (1, 520, 1365), (15, 128, 250), (16, 264, 64), (17, 64, 63),
           (63, 200, 130), (64, 136, 257), (65, 64, 512), (130, 328, 300), (257, 64, 1000), (300, 1024, 96)]


@pytest.mark.parametrize("T,d,d_ff", FORWARD)
@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
def test_forward(dtype, T, d, d_ff):
    layer = Layer(dtype, T, d, d_ff)
    kind = (T + d) % 3
    layer.check({"y": layer.forward(kind, d_ff % 2 == 1)}, kind, d_ff % 2 == 1)


@pytest.mark.parametrize("T,d,d_ff", [(1, 5, 3), (3, 67, 33), (70, 131, 100), (200, 515, 77)])
@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
def test_odd_widths(dtype, T, d, d_ff):
    """Rows that are no whole chunks."""
    layer = Layer(dtype, T, d, d_ff)
    layer.check(layer.train(2, True), 2, True)


BACKWARD = [(1, 8, 1), (1, 256, 300), (2, 64, 64), (16, 72, 130), (33, 264, 65), (64, 128, 200), (65, 520, 1365),
            (129, 64, 257), (300, 200, 512)]


@pytest.mark.parametrize("T,d,d_ff", BACKWARD)
@pytest.mark.parametrize("kind,silu", [(0, False), (1, True), (2, False)], ids=["relu", "rsplus_silu", "silu"])
@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
def test_training_step(dtype, kind, silu, T, d, d_ff):
    layer = Layer(dtype, T, d, d_ff, seed=kind)
    layer.check(layer.train(kind, silu), kind, silu)


@pytest.mark.parametrize("T,d,d_ff", [(2048, 72, 4100), (2050, 64, 2100), (1000, 64, 2000), (700, 1032, 8200),
                                      (4100, 520, 2600), (130, 4096, 14336)])
def test_large_tiles(T, d, d_ff):
    """Sizes that fill the chip with each of the bf16 tiles, and tokens' sums cut in shares."""
    layer = Layer(BF16, T, d, d_ff)
    layer.check(layer.train(1, False), 1, False)


@pytest.mark.parametrize("T,d,d_ff", [(1, 4096, 64), (5, 2048, 300), (16, 1032, 33), (33, 2048, 130), (64, 3000, 64),
                                      (70, 2048, 300), (200, 4096, 65), (2, 72, 3000)])
@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
def test_long_rows_in_few_tiles(dtype, T, d, d_ff):
    """Sums cut in shares in every product: the hidden layer's, dz's and the tokens' own."""
    layer = Layer(dtype, T, d, d_ff)
    layer.check(layer.train(1, True), 1, True)


@pytest.mark.parametrize("T,d,d_ff", [(6000, 72, 40), (9000, 136, 16), (4096, 8, 8), (5000, 64, 300)])
def test_gradients_over_many_tokens_of_small_layers(T, d, d_ff):
    """Weight gradients of a few tiles, their sums over tokens cut in shares."""
    for dtype in (BF16, F32):
        layer = Layer(dtype, T, d, d_ff)
        layer.check(layer.train(2), 2)


def test_one_workspace_for_many_calls():
    """Allocated for the most tokens, used for others in turn, forward and backward."""
    ws = ffn.alloc_gated_workspace(1500, 264, 700, BF16)
    for T in (1500, 1, 64, 65, 17, 300, 1000, 2):
        layer = Layer(BF16, T, 264, 700)
        layer.check(layer.train(2, ws=ws), 2, what=f"T={T}")


def test_two_calls_at_once():
    """Two streams, a workspace each."""
    layers = [Layer(BF16, T, 264, 900) for T in (40, 333)]
    sides = [torch.cuda.Stream() for _ in layers]
    bufs = [(torch.empty_like(a.x), ffn.alloc_gated_workspace(a.T, 264, 900, BF16)) for a in layers]
    torch.cuda.synchronize()
    for _ in range(5):
        for a, side, (y, ws) in zip(layers, sides, bufs):
            ffn.ffn_gated_forward(a.x, *a.w, a.t, ffn.options(act=2), y, ws, stream=side)
    torch.cuda.synchronize()
    for a, (y, _) in zip(layers, bufs):
        a.check({"y": y}, 2)


def test_paper_size_fp32():
    layer = Layer(F32, 130, 3840, 14231)
    layer.check(layer.train(2, True), 2, True)


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
def test_nothing_active(dtype):
    """A threshold above every gate value, infinity too: outputs and gradients are exact zeros."""
    for T in (1, 40, 200):
        layer = Layer(dtype, T, 72, 200)
        for t in (1e30, math.inf):
            for kind in (0, 1):
                for name, g in layer.train(kind, t=t).items():
                    assert not bool(g.any()), (T, t, kind, name)


def test_everything_active():
    layer = Layer(BF16, 70, 72, 200)
    layer.check(layer.train(0, t=-64.0), 0, t=-64.0)


@pytest.mark.parametrize("T", [5, 40, 150, 600])
def test_a_tokens_nan_is_its_own(T):
    """NaN and Inf of one token reach its rows of y and dx and no other's."""
    for dtype in (BF16, F32):
        layer = Layer(dtype, T, 136, 333)
        clean = layer.train(2)
        for bad, value in ((T // 2, math.nan), (T - 1, math.inf)):
            layer.x[bad, 3] = value
            got = layer.train(2)
            others = torch.arange(T, device="cuda") != bad
            for name in ("y", "dx"):
                assert torch.equal(got[name][others], clean[name][others]), (name, bad)
                assert not bool(torch.isfinite(got[name][bad]).all()), (name, bad)
            layer.x[bad, 3] = 0.0
            clean = layer.train(2)


def test_nan_gate_is_inactive():
    """A NaN gate value is not above the threshold: with the ReLU forms the neuron gives nothing."""
    for T in (1, 70):
        layer = Layer(F32, T, 64, 100)
        layer.w[0][7] = math.nan
        got = {k: layer.train(k) for k in (0, 1, 2)}
        for kind in (0, 1):
            assert bool(torch.isfinite(got[kind]["y"]).all())
            assert not bool(got[kind]["dw_gate"][7].any())
        assert bool(torch.isnan(got[2]["y"]).all())


@pytest.mark.parametrize("T,d,d_ff", [(3, 61, 70), (30, 130, 65), (100, 67, 129), (300, 260, 100)])
@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
def test_outputs_end_where_they_end(dtype, T, d, d_ff):
    """Every output lies between guards in one buffer; none is touched."""
    layer = Layer(dtype, T, d, d_ff)
    guard = 64

    def between(shape):
        n = shape[0] * shape[1]
        buf = torch.full((guard + n + guard,), 7.0, dtype=dtype, device="cuda")
        return buf, buf[guard:guard + n].view(shape)

    bufs = [between((T, d))] + [between((T, d))] + [between((d_ff, d)) for _ in range(3)]
    ws = ffn.alloc_gated_workspace(T, d, d_ff, dtype)
    size = ffn.alloc_gated_save(T, d_ff, dtype).numel()
    save = torch.full((size + 512,), 0x5A, dtype=torch.uint8, device="cuda")
    opt = ffn.options(act=2)
    ffn.ffn_gated_forward(layer.x, *layer.w, 0.25, opt, bufs[0][1], ws, save=save[:size])
    ffn.ffn_gated_backward(layer.x, *layer.w, opt, layer.dy, save[:size], *(b[1] for b in bufs[1:]), ws)
    for buf, view in bufs:
        assert bool((buf[:guard] == 7.0).all()) and bool((buf[-guard:] == 7.0).all())
    assert bool((save[size:] == 0x5A).all())
    layer.check(dict(zip(("y", "dx", "dw_gate", "dw_up", "dw_down_t"), (b[1] for b in bufs))), 2, t=0.25)


def test_some_gradients_only():
    layer = Layer(BF16, 90, 200, 300)
    full = layer.train(1)
    for k, name in enumerate(("dx", "dw_gate", "dw_up", "dw_down_t")):
        got = layer.train(1, want=[i == k for i in range(4)])
        assert torch.equal(got[name], full[name]), name


def test_same_bits_again():
    """No atomic adds: a second run gives the same bits, also where sums are cut in shares."""
    for T, d, d_ff in ((1, 512, 4096), (50, 256, 3000), (300, 520, 1365)):
        layer = Layer(BF16, T, d, d_ff)
        a, b = layer.train(1), layer.train(1)
        for name in a:
            assert torch.equal(a[name], b[name]), name


def test_save_serves_two_backward_calls():
    layer = Layer(F32, 40, 64, 100)
    save, ws = ffn.alloc_gated_save(40, 100, F32), ffn.alloc_gated_workspace(40, 64, 100, F32)
    layer.forward(2, save=save, ws=ws)
    opt, dx = ffn.options(act=2), [torch.empty_like(layer.x) for _ in range(2)]
    for out in dx:
        ffn.ffn_gated_backward(layer.x, *layer.w, opt, layer.dy, save, out, None, None, None, ws)
    assert torch.equal(*dx)


def test_other_stream_and_graph():
    """A training step on a side stream; captured, replayed on new tokens with eager work in between;
    two graphs that share a workspace, replayed in turn."""
    layer = Layer(BF16, 100, 136, 333)
    other = Layer(BF16, 100, 136, 333, seed=5)
    ws, save = ffn.alloc_gated_workspace(100, 136, 333, BF16), ffn.alloc_gated_save(100, 333, BF16)
    x, dy = layer.x.clone(), layer.dy.clone()
    opt = ffn.options(act=2)
    y, dx, dw = torch.empty_like(x), torch.empty_like(x), [torch.empty_like(w) for w in layer.w]

    def step():
        ffn.ffn_gated_forward(x, *layer.w, 0.0, opt, y, ws, save=save)
        ffn.ffn_gated_backward(x, *layer.w, opt, dy, save, dx, *dw, ws)

    def eager(xx, dyy):
        layer.x, layer.dy = xx, dyy
        return layer.train(2, t=0.0)

    want = [eager(layer.x, layer.dy), eager(other.x, other.dy)]
    inputs = [(x.clone(), dy.clone()), (other.x, other.dy)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    side.synchronize()
    assert torch.equal(y, want[0]["y"]) and torch.equal(dw[2], want[0]["dw_down_t"])
    graph, fwd = torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    y2 = torch.empty_like(y)
    with torch.cuda.graph(fwd):
        ffn.ffn_gated_forward(x, *layer.w, 0.0, opt, y2, ws)
    for r in (1, 0, 1):
        x.copy_(inputs[r][0])
        dy.copy_(inputs[r][1])
        for b in (y, dx, *dw, y2):
            b.fill_(math.nan)
        graph.replay()
        fwd.replay()
        torch.cuda.synchronize()
        got = dict(zip(("y", "dx", "dw_gate", "dw_up", "dw_down_t"), (y, dx, *dw)))
        for name in got:
            assert torch.equal(got[name], want[r][name]), (r, name)
        assert torch.equal(y2, want[r]["y"])
        assert torch.equal(eager(*inputs[r])["y"], want[r]["y"])


def test_stream_argument_and_refusals():
    layer = Layer(BF16, 8, 64, 100)
    ws, y = ffn.alloc_gated_workspace(8, 64, 100, BF16), torch.empty_like(layer.x)
    opt = ffn.options()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    ffn.ffn_gated_forward(layer.x, *layer.w, layer.t, opt, y, ws, stream=side)
    side.synchronize()
    layer.check({"y": y})
    g, u, dn = layer.w

    def call(x=layer.x, g=g, u=u, dn=dn, y=y, ws=ws, save=None):
        ffn.ffn_gated_forward(x, g, u, dn, 0.0, opt, y, ws, save=save)

    for bad in (dict(x=layer.x.float()), dict(g=g.float()), dict(u=u[:50]), dict(dn=dn[:, :32]), dict(y=y[:4]),
                dict(x=layer.x.t()), dict(g=None), dict(ws=ws.cpu()), dict(x=layer.x[0])):
        with pytest.raises((ValueError, TypeError)):
            call(**bad)
    with pytest.raises(ffn.FFNError):
        call(ws=ws[:256])
    with pytest.raises(ffn.FFNError):
        call(save=ws[:16])
    with pytest.raises(TypeError):
        call(x=layer.x.half())


def test_gradient_against_differences_of_the_kernel():
    """(L(x + e p) - L(x - e p)) / 2e of the fp32 block's own outputs, L = <y, dy>, against <dx, p>.  The two
    outputs are off by at most the forward bound of their norm each; the difference's own truncation is
    taken from the same quotient in 64 bits."""
    T, d, d_ff, e = 24, 64, 160, 2.0 ** -5
    layer = Layer(F32, T, d, d_ff)
    dx = layer.train(2, True, t=0.0)["dx"].double()
    gen = torch.Generator(device="cuda").manual_seed(1)
    p = torch.randn((T, d), generator=gen, device="cuda")
    dy, x = layer.dy.double(), layer.x.clone()
    L, exact, noise = [], [], 0.0
    for s in (e, -e):
        xs = x + s * p
        y = layer.forward(2, True, t=0.0, x=xs).double()
        ys = ref.forward(xs, *layer.w, 0.0, 2, True)["y"]
        L.append(float((y * dy).sum()))
        exact.append(float((ys * dy).sum()))
        noise += ref.bound(F32, 8, d + d_ff) * float(ys.norm()) * float(dy.norm()) / (2 * e)
    # x + e p itself rounds: the same xs went to both sides
    ref_dx = layer.reference(2, True, t=0.0)["dx"]
    truncation = abs((exact[0] - exact[1]) / (2 * e) - float((ref_dx * p.double()).sum()))
    bound_dx = ref.bound(F32, 8, 2 * (d + d_ff)) * float(ref_dx.norm()) * float(p.double().norm())
    assert abs((L[0] - L[1]) / (2 * e) - float((dx * p.double()).sum())) <= noise + truncation + bound_dx


def test_offsets_past_32_bits():
    """600000 tokens: g, v and z pass 2^31 bytes.  A few tokens are compared, the last among them."""
    T, d, d_ff = 600000, 8, 1000
    layer = Layer.__new__(Layer)
    gen = torch.Generator(device="cuda").manual_seed(2)
    layer.dtype, layer.T, layer.d, layer.d_ff, layer.t = BF16, T, d, d_ff, 0.25
    layer.x = torch.randn((T, d), generator=gen, device="cuda").to(BF16)
    layer.dy = torch.randn((T, d), generator=gen, device="cuda").to(BF16)
    layer.w = [(torch.randn((d_ff, d), generator=gen, device="cuda") * s).to(BF16) for s in (0.35, 0.35, 0.03)]
    got = layer.train(2)
    at = torch.tensor([0, 1, 255, 262144, 524288, 599744, 599998, 599999], device="cuda")
    part = Layer.__new__(Layer)
    part.__dict__.update(layer.__dict__, T=len(at), x=layer.x[at].contiguous(), dy=layer.dy[at].contiguous())
    want = part.reference(2)
    ref.check(got["y"][at], want["y"], BF16, 2, d + d_ff, "y")
    ref.check(got["dx"][at], want["dx"], BF16, 2, 2 * (d + d_ff), "dx")
    # the weight gradients: sums over all tokens, in 64 bits by pieces
    total = None
    for k in range(0, T, 50000):
        part.__dict__.update(x=layer.x[k:k + 50000], dy=layer.dy[k:k + 50000])
        r = part.reference(2)
        total = {n: r[n] if total is None else total[n] + r[n] for n in r if n.startswith("dw")}
    for n in ("dw_gate", "dw_up", "dw_down_t"):
        ref.check(got[n], total[n], BF16, 2, T + 2 * d, n)


def test_agrees_with_the_decode_calls():
    """One layer through the block and through the decode calls' dense and sparse forms (fp32 weights)."""
    T, d, d_ff = 6, 512, 2048
    layer = Layer(F32, T, d, d_ff, near=1.28)
    y = layer.forward()
    ws = ffn.alloc_workspace(T, d, d_ff)
    for call in (ffn.ffn_dense_forward, ffn.ffn_sparse_forward):
        z = torch.empty_like(y)
        call(layer.x, *layer.w, layer.t, z, ws)
        assert float((z - y).norm()) <= 2 * ref.bound(F32, 8, d + d_ff) * float(y.norm())


def test_a_layer_trained_and_then_served():
    """Steps of gradient descent with the block's gradients lower the loss that they are the gradient of to
    first order, and the layer then runs in the sparse decode call as in the block."""
    T, d, d_ff, rate = 64, 128, 512, 2.0 ** -10
    layer = Layer(F32, T, d, d_ff, near=1.0)
    want = layer.reference(1)
    target = layer.dy
    for _ in range(3):
        save, ws = ffn.alloc_gated_save(T, d_ff, F32), ffn.alloc_gated_workspace(T, d, d_ff, F32)
        y = layer.forward(1, save=save, ws=ws)
        layer.dy = (y - target).contiguous()
        dw = [torch.empty_like(w) for w in layer.w]
        ffn.ffn_gated_backward(layer.x, *layer.w, ffn.options(act=1), layer.dy, save, None, *dw, ws)
        layer.check(dict(zip(("dw_gate", "dw_up", "dw_down_t"), dw)), 1)
        layer.w = [(w - rate * g).contiguous() for w, g in zip(layer.w, dw)]
        layer.t = ref.threshold_in_gap(layer.x.double() @ layer.w[0].double().t(), 1.0)
    y = layer.forward(1)
    z, ws = torch.empty_like(y), ffn.alloc_workspace(T, d, d_ff)
    ffn.ffn_sparse_forward_ex(layer.x, *layer.w, layer.t, ffn.options(act=1), z, ws)
    assert float((z - y).norm()) <= 2 * ref.bound(F32, 8, d + d_ff) * float(y.norm())
    assert want["y"].shape == y.shape
