"""The precision of layer norm's dweight and dbias where they are summed beside dX."""
import sys

import pytest
import torch

import dense_util as du
from test_gpu_layer_norm import operands

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def lut():
    import paper_2302_03213_amd as lut_mod
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    return lut_mod


@pytest.fixture(autouse=True)
def announce(request):
    print("\n[case] %s" % request.node.nodeid, file=sys.stderr, flush=True)
    yield


@pytest.mark.parametrize("kind", list(du.TYPES))
@pytest.mark.parametrize("N,D", [(1, 40), (17, 3), (600, 768), (1024, 1000), (700, 4099), (768, 2048), (333, 16384)])
def test_sums_beside_dx_are_64_bit_ones(lut, N, D, kind):
    """dbias is the exact sum rounded once; dweight is off by its terms' own (x - mean) rstd, each by 2 u, and one rounding."""
    X, _, G, w, _ = operands(N, D, du.TYPES[kind], seed=N + D, shift=0.5)
    statistics = torch.empty((N, 2), device="cuda")
    lut.layer_norm(X, statistics=statistics)
    with lut.tunables(LUTNN_NORM_SUMS="beside"):
        _, dw, db = lut.layer_norm_backward(G, X, statistics, w)
    g, h = G.double(), (X.double() - statistics[:, :1].double()) * statistics[:, 1:].double()
    exact = 1024 * 2.0 ** -53  # of as many additions in 64 bits, relative to the sum of sizes
    du.check(db, g.sum(0), du.U * g.sum(0).abs() + exact * g.abs().sum(0))
    du.check(dw, (g * h).sum(0), du.U * (g * h).sum(0).abs() + (2.01 * du.U + exact) * (g * h).abs().sum(0))
