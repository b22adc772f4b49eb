"""The norms' gradients that are summed over the tokens, held to the chains of additions that the backward call makes."""
import pytest

from tests import norm_ref as ref
from tests.norm_chains import chain
from tests.test_gpu_norm import BF16, F32, KINDS, Layer

pytestmark = pytest.mark.gpu

# a row a group, two, more than are in flight at once; each count of threads to a row
SIZES = [(1, 64), (3, 512), (7, 300), (2048, 24), (2049, 24), (5001, 100), (128, 520), (300, 1001), (1025, 520), (2049, 1040), (5000, 2048),
         (128, 2056), (700, 4096), (3001, 2500), (129, 4104), (300, 4104), (515, 8192), (1100, 5001), (257, 9000), (40, 16384)]


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("kind", ["row", "no_gains", "token"])
@pytest.mark.parametrize("T,d", SIZES)
def test_sums_over_the_tokens(dtype, kind, T, d):
    layer = Layer(dtype, T, d, **KINDS[kind])
    o = layer.run()
    rf, r = (o["rstd"][i].double()[:, None] for i in (0, 1))
    want, err = ref.backward(o["x_out"], layer.f, layer.ref, rf, r, layer.dn, layer.dxo, chain(T, d))
    for name in ("dpre_gain", "dpost_gain") + (("dgate",) if layer.gate.shape[0] == 1 else ()):
        ref.check(o[name], want[name], err[name], dtype, f"{kind} T={T} d={d} {name}")
