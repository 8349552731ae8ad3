"""What the gradients of 16-bit dense layers are rounded by: once where dZ is a value of the type anyway, twice where a slope makes it."""
import sys

import pytest
import torch

import dense_util as du
from test_gpu_dense_linear import operands

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


def off(got, want):
    return ((got.double() - want).norm() / want.norm()).item()


# One rounding to nearest, in the 2-norm: the error is uniform within half a step, and half a step is half(T) / m of a value whose
# significand m is spread over [1, 2) as 1 / m: half(T) sqrt(1/3 * 3 / (8 ln 2)) = 0.425 half(T).  Over 10^5 values and more the
# sampled norm is within 1 % of that; significands spread otherwise move it by 3 %.
def once(T):
    return 0.425 * du.half(T) * 1.05


@pytest.mark.parametrize("kind", ["bf16", "f16"])
@pytest.mark.parametrize("N,D,M", [(700, 264, 520), (2000, 768, 768), (4100, 4104, 4104)])
def test_roundings(lut, N, D, M, kind):
    T = du.TYPES[kind]
    X, W, _, _, G = operands(N, D, M, T, seed=N)
    Z = du.random((N, M), T, seed=5, scale=2)
    for activation in du.ACTIVATIONS:
        dz = G.double() * (1 if activation is None else du.slope64(Z.double(), activation))
        dX, dW, db = lut.dense_linear_backward(X, W, G, Z if activation else None, activation)
        allowed = once(T) * (1 if activation in (None, "relu") else 2 ** 0.5)
        assert off(dX, dz @ W.double().t()) <= allowed and off(dW, X.double().t() @ dz) <= allowed, activation
        # dbias has none of them: a slope is off by a few u, and its sums by less
        assert off(db, dz.sum(0)) <= 8 * du.U, activation


def test_the_same_gradients_every_time(lut):
    """The largest timed layer: no pass differs from another in any bit, with other work between them."""
    X, W, _, _, G = operands(8192, 4096, 4096, torch.bfloat16, seed=1)
    Z, other = du.random((8192, 4096), torch.bfloat16, seed=2), operands(1000, 515, 1030, torch.bfloat16, seed=3)
    first = lut.dense_linear_backward(X, W, G, Z, "gelu_tanh")
    for _ in range(8):
        lut.dense_linear_backward(other[0], other[1], other[4])
        for a, b in zip(lut.dense_linear_backward(X, W, G, Z, "gelu_tanh"), first):
            assert torch.equal(a, b)
