"""Operands near both ends of the range and values that are not finite, by every form of the dense layers' products, pinned.  dense_util.py
derives the tolerances."""
import sys

import pytest
import torch

import dense_forms as df
import dense_util as du
from test_gpu_dense_linear import operands

pytestmark = pytest.mark.gpu

PINNED = [(kind, form, splits) for kind in du.TYPES for form in df.FORMS[kind] for splits in (1, 3) if form != "memory" or splits == 1]
PLANES = [(form, splits) for form in ("128x256", "128x128") for splits in (1, 3)]


@pytest.fixture(scope="module")
def lut():
    import paper_2302_03213_amd as lut_mod
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    return lut_mod


@pytest.fixture(autouse=True)
def announce(request):
    print("\n[case] %s" % request.node.nodeid, file=sys.stderr, flush=True)
    yield


def pin(lut, form, splits):
    return lut.tunables(LUTNN_DENSE_FORM=form, LUTNN_DENSE_SPLITS=splits)


@pytest.mark.parametrize("form,splits", PLANES)
@pytest.mark.parametrize("x_up,w_up", [(-60, 30), (50, 40), (110, -100), (-100, 110), (60, -60)])
def test_fp32_sums_of_values_of_any_size(lut, form, splits, x_up, w_up):
    """Operands and products whose parts leave the range are summed another way."""
    X, W, _, _, G = operands(150, 200, 520, torch.float32, seed=8)
    X, W = X * 2.0 ** x_up, W * 2.0 ** w_up
    with pin(lut, form, splits):
        y, y_off, _, _ = du.dense64(X, W)
        du.check(lut.dense_linear(X, W), y, y_off)
        Z = du.random(G.shape, torch.float32, 9)
        for g, (want, off) in zip(lut.dense_linear_backward(X, W, G, Z, "silu"), du.dense_backward64(X, W, G, Z, "silu")):
            du.check(g, want, off)


def check_where_finite(got, want, off):
    """The same entries missing and infinite, with the same signs, as in 64 bits; the others within `off`."""
    got = got.double()
    assert torch.isnan(got).equal(torch.isnan(want)) and torch.isinf(got).equal(torch.isinf(want))
    assert torch.equal(got[torch.isinf(got)], want[torch.isinf(got)])
    fine = torch.isfinite(want)
    du.check(got[fine], want[fine], off[fine])


def without(t):
    return torch.where(torch.isfinite(t), t, torch.zeros_like(t))


@pytest.mark.parametrize("kind,form,splits", PINNED)
@pytest.mark.parametrize("pad", [0, 5])
def test_values_that_are_not_finite(lut, kind, form, splits, pad):
    """They reach the sums that they are in and no others, with strides and in front of an activation's slope too."""
    T, (N, D, M) = du.TYPES[kind], (290, 136, 300)
    X, W, b, R, G = operands(N, D, M, T, seed=21)
    Z = du.random((N, M), T, seed=6)
    X[2, 7], X[140, 130], W[5, 11], W[100, 290] = float("inf"), float("nan"), float("-inf"), float("inf")
    G[3, 9], G[200, 299], G[289, 0] = float("inf"), float("-inf"), float("nan")
    x, w, g, z = (du.strided(t, pad) if pad else t for t in (X, W, G, Z))
    with pin(lut, form, splits):
        # the errors of what is finite are those of operands without the others: no finite sum has one in it
        off = du.dense64(without(X), without(W), b)[1]
        check_where_finite(lut.dense_linear(x, w, b), X.double() @ W.double() + b.double(), off)
        for activation in (None, "gelu", "relu"):
            offs = [o for _, o in du.dense_backward64(without(X), without(W), without(G), Z, activation)]
            dz = G.double() * (1 if activation is None else du.slope64(Z.double(), activation))
            wanted = dz @ W.double().t(), X.double().t() @ dz, dz.sum(0)
            for needs in ((True, True, True), (True, False, False), (False, True, False)):
                for got, want, o in zip(lut.dense_linear_backward(x, w, g, z if activation else None, activation, *needs), wanted, offs):
                    if got is not None:
                        check_where_finite(got, want, o)
