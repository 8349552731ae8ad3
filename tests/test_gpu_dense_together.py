"""The dense layers and norms with the table-lookup layers, as a transformer's feed-forward half uses them: modules chained in a training
step against the same step made of single calls, bit for bit, and against 64 bits where no lookup is in the way."""
import sys

import pytest
import torch

import dense_util as du

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


def test_a_block_with_a_looked_up_layer(lut):
    """norm -> dense with gelu -> table lookup, then the residual's norm: the first half dense, the second looked up."""
    from paper_2302_03213_amd import binding
    from paper_2302_03213_amd.dense import DenseLinear, LayerNorm
    from paper_2302_03213_amd.softpq import SoftPQLinear
    N, D, H, V = 300, 64, 256, 4
    X, G = du.random((N, D), torch.float32, 1), du.random((N, D), torch.float32, 2)
    W1, b1 = du.random((D, H), torch.float32, 3, D ** -0.5), du.random((H,), torch.float32, 4, 0.1)
    W2, b2 = du.random((H, D), torch.float32, 5, H ** -0.5), du.random((D,), torch.float32, 6, 0.1)
    centroids = du.random((H // V, 16, V), torch.float32, 7, 0.5)
    first, up, last = LayerNorm(D), DenseLinear(W1, b1, "gelu"), LayerNorm(D)
    down = SoftPQLinear(centroids, W2, b2)
    x = X.clone().requires_grad_()
    out = last(down(up(first(x))), residual=x)
    out.backward(G)

    # the same by single calls
    s1, s2 = (torch.empty((N, 2), device="cuda") for _ in range(2))
    Z, total = torch.empty((N, H), device="cuda"), torch.empty_like(X)
    normed = lut.layer_norm(X, first.weight, first.bias, statistics=s1)
    hidden = lut.dense_linear(normed, W1, b1, "gelu", preactivation=Z)
    looked_up = lut.linear(lut.build_table(centroids, W2, lut.TABLE_I8, bias=b2), hidden)
    y = lut.layer_norm(looked_up, last.weight, last.bias, residual=X, total=total, statistics=s2)
    assert torch.equal(out, y)
    dsum, dw2, db2 = lut.layer_norm_backward(G, total, s2, last.weight)
    dP, dhidden, dt = binding._softpq_gradients(centroids, D, 1.0, hidden, binding._input_gradient(dsum, W2), True)
    dnormed, dW1, db1 = lut.dense_linear_backward(normed, W1, dhidden, Z, "gelu")
    dx, dw1, dbn = lut.layer_norm_backward(dnormed, X, s1, first.weight)
    for got, want in ((last.weight.grad, dw2), (last.bias.grad, db2), (down.centroids.grad, dP), (up.W.grad, dW1), (up.bias.grad, db1),
                      (first.weight.grad, dw1), (first.bias.grad, dbn), (down.temperature.grad, dt.reshape(()))):
        assert torch.equal(got, want)
    assert torch.equal(x.grad, dx + dsum) or torch.equal(x.grad, dsum + dx)


@pytest.mark.parametrize("kind", list(du.TYPES))
def test_a_dense_block(lut, kind):
    """Pre-norm feed-forward blocks, forward and backward, against 64 bits."""
    from paper_2302_03213_amd.dense import DenseLinear, LayerNorm
    T, N, D, H = du.TYPES[kind], 200, 64, 256
    X, G = du.random((N, D), T, 1), du.random((N, D), T, 2)
    W = [du.random(shape, T, 3 + i, shape[0] ** -0.5) for i, shape in enumerate(((D, H), (H, D)))]
    b = [du.random((n,), torch.float32, 6 + i, 0.1) for i, n in enumerate((H, D))]
    norm, up, down, last = LayerNorm(D), DenseLinear(W[0], b[0], "gelu_tanh"), DenseLinear(W[1], b[1]), LayerNorm(D)
    x = X.clone().requires_grad_()
    y, total = last(down(up(norm(x))), residual=x, with_total=True)
    torch.autograd.backward([y, total], [G, G])

    f = torch.nn.functional
    x64 = X.double().requires_grad_()
    w64 = [w.double().requires_grad_() for w in W]
    h = f.gelu(f.layer_norm(x64, (D,), eps=1e-5) @ w64[0] + b[0].double(), approximate="tanh")
    total64 = h @ w64[1] + b[1].double() + x64
    y64 = f.layer_norm(total64, (D,), eps=1e-5)
    torch.autograd.backward([y64, total64], [G.double(), G.double()])
    # Five stages forward and five back.  Each rounds its result to T by half a step and has an fp32 sum's error of at most H terms
    # in it; none makes an error of its input larger than fourfold, relative to the largest value of its result (weights that keep the
    # size, rows of spread about one, slopes below 1.13), and the errors of ten stages add up.
    per_stage = du.half(T) + du.sum_error(H)
    for got, want in ((y, y64), (total, total64), (x.grad, x64.grad), (up.W.grad, w64[0].grad), (down.W.grad, w64[1].grad)):
        assert (got.double() - want).abs().max() <= 10 * 4 * per_stage * want.abs().max()
