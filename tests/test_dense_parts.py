"""The arithmetic behind the bound that single fp32 products are held to (test_gpu_dense_precision.py).  No GPU needed."""
import numpy as np

import dense_forms as df


def parts(x):
    """An fp32 value as three bf16 ones: the top eight significant bits, the next eight, the rest."""
    def cut(v):
        return (v.view(np.uint32) & np.uint32(0xffff0000)).view(np.float32)
    x = x * np.float32(2.0 ** 24)
    r = x - cut(x)
    return [p.astype(np.float64) for p in (cut(x), cut(r), cut(r - cut(r)))]


def test_the_bound_of_one_term_notices_every_product():
    """What is left of a product without any one of the six lies outside the bound; all six lie within the part of it that they may use."""
    rng = np.random.default_rng(0)
    a, b = (rng.standard_normal(4096).astype(np.float32) for _ in range(2))
    (h, m, l), (g, n, k) = parts(a), parts(b)
    six = [l * g, h * k, m * n, m * g, h * n, h * g]
    exact = a.astype(np.float64) * b.astype(np.float64)

    def off(terms):
        return (np.abs(sum(terms) * 2.0 ** -48 - exact) / np.abs(exact)).max()

    assert off(six) <= 2.0 ** -21 * (1 + 2.0 ** -8)
    for i in range(6):
        assert off(six[:i] + six[i + 1:]) > 8 * df.ONE_TERM, i
