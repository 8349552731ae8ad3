"""Single fp32 products by every form of the dense layers, pinned: whether all their parts' products are there.  dense_forms.py derives the
bound."""
import sys

import pytest
import torch

import dense_forms as df
import dense_util as du

pytestmark = pytest.mark.gpu

PINNED = [(form, splits) for form in df.FORMS["f32"] for splits in (1, 3) if form != "memory" or splits == 1]


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


@pytest.mark.parametrize("form,splits", PINNED)
@pytest.mark.parametrize("N,D,M", [(300, 264, 520), (130, 1000, 257), (520, 31, 300)])
@pytest.mark.parametrize("up", [0, -100, 90])
def test_fp32_products_keep_fp32_precision(lut, form, splits, N, D, M, up):
    """Sums that have one term each: what is left of that product without any of the parts' six is outside the bound
    (test_dense_parts.py).  Also of operands near both ends of the range."""
    X, at = df.one_per_row(N, D, 1)
    W, G = du.random((D, M), torch.float32, 2), du.random((N, M), torch.float32, 3)
    X, W = X * 2.0 ** up, W * 2.0 ** -up
    with pin(lut, form, splits):
        df.check_relative(lut.dense_linear(X, W), X[torch.arange(N), at].double()[:, None] * W.double()[at], df.ONE_TERM)
        sparse, at = df.one_per_row(N, M, 4)
        dx = (sparse * 2.0 ** up)[torch.arange(N), at].double()[:, None] * W.double()[:, at].t()
        columns, rows = df.one_per_row(D, N, 5)
        columns = columns.t().contiguous() * 2.0 ** up
        dw = columns[rows, torch.arange(D)].double()[:, None] * (G * 2.0 ** -up).double()[rows]
        for both in (True, False):
            df.check_relative(lut.dense_linear_backward(columns, W, sparse * 2.0 ** up, need_dw=both)[0], dx, df.ONE_TERM)
            df.check_relative(lut.dense_linear_backward(columns, W, G * 2.0 ** -up, need_dx=both)[1], dw, df.ONE_TERM)
