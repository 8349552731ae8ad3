"""Layer norm's gradients by every way that dweight and dbias are summed, pinned by the switch LUTNN_NORM_SUMS, at widths of every kernel
and at more rows than it has workgroups: against 64 bits and bit for bit against themselves.  dense_util.py derives the tolerances."""
import sys

import pytest
import torch

import dense_util as du
from test_gpu_layer_norm import EPS, operands

pytestmark = pytest.mark.gpu

SUMS = ("beside", "1", "2")
# rows that end with a vector moved back and that do not, for 16 threads a row to 1024, fewer rows than workgroups and more
SIZES = [(1025, 1025), (1030, 2049), (1100, 4095), (1100, 4096), (2050, 3001), (1100, 5121), (1030, 16383), (600, 8192), (1030, 9000),
         (1300, 768), (40, 3000), (3000, 33), (5, 16384), (1, 1025), (2000, 5), (530, 264)]


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
@pytest.mark.parametrize("sums", SUMS + (None,))
@pytest.mark.parametrize("N,D", SIZES)
def test_backward(lut, N, D, sums, kind):
    X, R, G, w, b = operands(N, D, du.TYPES[kind], seed=N + D)
    statistics = torch.empty((N, 2), device="cuda")
    lut.layer_norm(X, statistics=statistics)
    with lut.tunables(LUTNN_NORM_SUMS=sums):
        for weight, residual in ((w, None), (w, R), (None, None)):
            got = lut.layer_norm_backward(G, X, statistics, weight, residual)
            wanted = du.norm_backward64(G, X, statistics, weight, residual)
            for g, want in zip(got, wanted):
                du.check(g, *want)
            for needs in ((True, False, False), (False, True, True), (True, True, False), (False, False, True), (True, True, True)):
                parts = lut.layer_norm_backward(G, X, statistics, weight, residual, *needs)
                for needed, part, whole, want in zip(needs, parts, got, wanted):
                    if not needed:
                        assert part is None
                    elif sums is None:  # what is read decides how many workgroups share the rows
                        du.check(part, *want)
                    else:
                        assert torch.equal(part, whole)


@pytest.mark.parametrize("kind", list(du.TYPES))
@pytest.mark.parametrize("sums", SUMS)
@pytest.mark.parametrize("N,D", [(1030, 1001), (600, 4099), (300, 16380)])
def test_strides(lut, N, D, sums, kind):
    X, R, G, w, b = operands(N, D, du.TYPES[kind], seed=6)
    x, r, g = (du.strided(t, 3, 5) for t in (X, R, G))
    statistics = torch.empty((N, 2), device="cuda")
    lut.layer_norm(X, statistics=statistics)
    with lut.tunables(LUTNN_NORM_SUMS=sums):
        for a, c in zip(lut.layer_norm_backward(g, x, statistics, w, r), lut.layer_norm_backward(G, X, statistics, w, R)):
            assert torch.equal(a, c)


@pytest.mark.parametrize("sums", SUMS)
def test_captured(lut, sums):
    X, R, G, w, b = operands(1200, 2050, torch.bfloat16, seed=4)
    statistics, total = torch.empty((1200, 2), device="cuda"), torch.empty_like(X)

    def step():
        Y = lut.layer_norm(X, w, b, EPS, R, total=total, statistics=statistics)
        return (Y, total, statistics, *lut.layer_norm_backward(G, total, statistics, w, G))

    with lut.tunables(LUTNN_NORM_SUMS=sums):
        step()
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            captured = step()
        for seed in (31, 32, 33):
            for t, n in zip((X, R, G, w, b), operands(1200, 2050, torch.bfloat16, seed)):
                t.copy_(n)
            graph.replay()
            torch.cuda.synchronize()
            held = [t.clone() for t in captured]
            for a, c in zip(held, step()):
                assert torch.equal(a, c)
