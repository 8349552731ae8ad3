"""Layer norm's gradients from the total that the forward pass kept, which is rounded to its type, beside statistics of what was not."""
import sys

import pytest
import torch

import dense_util as du
from test_gpu_layer_norm import EPS, operands

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def announce(request):
    print("\n[case] %s" % request.node.nodeid, file=sys.stderr, flush=True)
    yield


@pytest.mark.parametrize("kind", list(du.TYPES))
@pytest.mark.parametrize("N,D,shift", [(50, 264, 0.0), (50, 264, 30.0), (1100, 1032, 30.0), (40, 3001, 100.0), (300, 768, 3.0)])
def test_module_gradients_of_rows_far_from_zero(kind, N, D, shift):
    """Against the gradients of the unrounded sum's norm: off by what the total's rounding is against the row's spread, and no more."""
    from paper_2302_03213_amd.dense import LayerNorm
    T, U = du.TYPES[kind], du.U
    X, R, G, w, b = operands(N, D, T, seed=N + D, shift=shift)
    G2 = du.random((N, D), T, 77)
    norm = LayerNorm(D, EPS)
    with torch.no_grad():
        norm.weight.copy_(w)
        norm.bias.copy_(b)
    x, r = X.clone().requires_grad_(), R.clone().requires_grad_()
    Y, total = norm(x, r, with_total=True)
    torch.autograd.backward([Y, total], [G, G2])
    assert torch.equal(x.grad, r.grad) and x.grad.data_ptr() != r.grad.data_ptr()

    s, g = X.double() + R.double(), G.double()
    y, (_, total_off), (mean, mean_off), (rstd, rstd_off) = du.norm64(X, w, b, EPS, R)
    du.check(Y.detach(), *y)
    du.check(total.detach(), s, total_off)
    h, q = (s - mean) * rstd, g * w.double()
    c, ch = q.mean(1, keepdim=True), (q * h).mean(1, keepdim=True)
    dx = rstd * (q - c - h * ch) + G2.double()
    # h from the rounded total and the statistics as they are; then as in dense_util.norm_backward64, with what h is off by squared too
    rel = rstd_off / rstd
    h_off = rstd * (total_off + mean_off) + h.abs() * rel + 3 * U * (s.abs() + mean.abs()) * rstd
    c_off = 46 * U * q.abs().mean(1, keepdim=True)
    ch_off = 46 * U * (q * h).abs().mean(1, keepdim=True) + (q.abs() * h_off).mean(1, keepdim=True)
    dx_off = rstd * (c_off + h.abs() * ch_off + h_off * (ch.abs() + ch_off) + 6 * U * (q.abs() + c.abs() + (h * ch).abs()))
    dx_off = dx_off + (dx - G2.double()).abs() * rel + 2 * U * dx.abs()
    du.check(x.grad, dx, dx_off * (1 + du.half(T)) + du.half(T) * dx.abs() + du.smallest(T))
    terms = (N / 256 + 20) * U
    du.check(norm.weight.grad, (g * h).sum(0), terms * (g * h).abs().sum(0) + (g.abs() * h_off).sum(0) * (1 + terms))
    du.check(norm.bias.grad, g.sum(0), terms * g.abs().sum(0))
