"""Shared by the tests of the dense linear layer and of layer norm: inputs, 64-bit references and the errors that fp32 sums and one
rounding to the result's type may leave.

u = 2^-24 is half a step of fp32, half(T) half a step of T, both relative to the value."""
import math

import torch

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
ACTIVATIONS = (None, "relu", "gelu", "gelu_tanh", "silu")
U = 2.0 ** -24


def half(T):
    return torch.finfo(T).eps / 2


def smallest(T):
    """Half the distance of the smallest values: what rounding is off by where half(T) times the value is less."""
    return torch.finfo(T).smallest_normal * torch.finfo(T).eps / 2


def random(shape, T, seed, scale=1.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(shape, generator=g) * scale).to(T).cuda()


def strided(t, pad, shift=0):
    """The same matrix with `pad` more values per row, `shift` values behind the start of its memory."""
    N, D = t.shape
    wide = torch.full((N * (D + pad) + shift,), float("nan"), dtype=t.dtype, device=t.device)
    view = wide[shift:].view(N, D + pad)[:, :D]
    view.copy_(t)
    return view


def act64(z, kind):
    f = torch.nn.functional
    return {None: lambda v: v, "relu": f.relu, "gelu": f.gelu, "silu": f.silu,
            "gelu_tanh": lambda v: f.gelu(v, approximate="tanh")}[kind](z)


def slope64(z, kind):
    z = z.detach().clone().requires_grad_()
    return torch.autograd.grad(act64(z, kind).sum(), z)[0]


def check(got, want, tolerance):
    """got within `tolerance` (a tensor) of the 64-bit `want`; the worst share of it, for the message."""
    got, want = got.double(), want.double()
    assert got.shape == want.shape
    assert torch.isfinite(got).all()
    worst = ((got - want).abs() / tolerance.clamp_min(1e-300)).max().item() if got.numel() else 0.0
    assert worst <= 1.0, "off by %.3g of what is allowed" % worst


def sum_error(terms):
    """Of an fp32 sum of `terms` products, relative to the sum of their sizes: an addition may be off by u, or by 2 u where it is
    cut instead of rounded, as in the matrix instructions, and a product from bf16 parts by 2^-21 = 8 u."""
    return (2 * terms + 16) * U


def dense64(X, W, bias=None, activation=None, residual=None):
    """Y, Z and what each may be off by."""
    T, D = X.dtype, X.shape[1]
    x, w = X.double(), W.double()
    z, size = x @ w, x.abs() @ w.abs()
    if bias is not None:
        z, size = z + bias.double(), size + bias.double().abs()
    z_off = sum_error(D) * size
    y = act64(z, activation)
    # no activation is steeper than 1.13; each is computed by a few fp32 operations on values up to z, exp among them, whose
    # argument's rounding weighs by its size: 2^-20 (|z| + 1) is 16 of them
    y_off = 1.13 * z_off + (0 if activation in (None, "relu") else 2.0 ** -20 * (z.abs() + 1))
    if residual is not None:
        y = y + residual.double()
        y_off = y_off + U * y.abs()
    return (y, y_off * (1 + half(T)) + half(T) * y.abs() + smallest(T),
            z, z_off * (1 + half(T)) + half(T) * z.abs() + smallest(T))


def dense_backward64(X, W, G, Z, activation):
    T, (N, M) = X.dtype, G.shape
    x, w, g = X.double(), W.double(), G.double()
    dz = g if activation is None else g * slope64(Z.double(), activation)
    # the slope as the activation above; dZ is rounded to T before it is multiplied
    off = torch.zeros_like(g) if activation is None else g.abs() * 2.0 ** -20 * (Z.double().abs() + 1)
    rounded = off if activation is None else off * (1 + half(T)) + half(T) * dz.abs() + smallest(T)

    def outer(value, size, terms, by_off):
        return value, (sum_error(terms) * size + by_off) * (1 + half(T)) + half(T) * value.abs() + smallest(T)

    dX = outer(dz @ w.t(), dz.abs() @ w.abs().t(), M, rounded @ w.abs().t())
    dW = outer(x.t() @ dz, x.abs().t() @ dz.abs(), N, x.abs().t() @ rounded)
    db = dz.sum(dim=0), sum_error(N) * dz.abs().sum(dim=0) + off.sum(dim=0)
    return dX, dW, db


def norm64(X, weight, bias, eps, residual):
    """Y, the sum, mean and rstd, each with what it may be off by."""
    T, (N, D) = X.dtype, X.shape
    s = X.double() + (0 if residual is None else residual.double())
    w = torch.ones(D, dtype=torch.float64, device=X.device) if weight is None else weight.double()
    b = torch.zeros(D, dtype=torch.float64, device=X.device) if bias is None else bias.double()
    mean = s.mean(dim=1, keepdim=True)
    far = s - mean
    rstd = (far.square().mean(dim=1, keepdim=True) + eps).rsqrt()
    h = far * rstd
    y = h * w + b
    # a row's sums: 16 values in a thread, ten steps over threads, sixteen wavefronts' sums: 42 additions, each off by u of the
    # sum of sizes.  The differences from a mean that is off by m are off by m + u |s|; their squares' sum is off by the square
    # of that on average, as far as the differences add up to nothing
    m = 42 * U * s.abs().mean(dim=1, keepdim=True)
    m = m + U * mean.abs()
    far_off = m + 2 * U * s.abs()
    # relative error of rstd: half of the variance's, and its own few roundings; the differences' own errors add what each is off
    # by, weighed by the difference
    rstd_off = (0.5 * (48 * U) + rstd.square() * ((far.abs() * 2 * U * s.abs()).mean(dim=1, keepdim=True) + m.square())) + 4 * U
    y_off = w.abs() * (rstd * far_off + h.abs() * (rstd_off + 4 * U)) + 2 * U * (y.abs() + b.abs())
    total_off = half(T) * s.abs() * (1 + 2 * U) + U * s.abs() + smallest(T)
    return ((y, y_off * (1 + half(T)) + half(T) * y.abs() + smallest(T)), (s, total_off),
            (mean, m), (rstd, rstd * rstd_off))


def norm_backward64(G, X, statistics, weight, residual):
    T, (N, D) = X.dtype, X.shape
    g, x, r = G.double(), X.double(), 0 if residual is None else residual.double()
    mean, rstd = statistics[:, :1].double(), statistics[:, 1:].double()
    w = torch.ones(D, dtype=torch.float64, device=X.device) if weight is None else weight.double()
    h, q = (x - mean) * rstd, g * w
    c, ch = q.mean(dim=1, keepdim=True), (q * h).mean(dim=1, keepdim=True)
    dx = rstd * (q - c - h * ch) + r
    # h is off by 3 u of (|x| + |mean|) rstd; the row's means as the sums of norm64, 42 additions and a few roundings
    h_off = 3 * U * (x.abs() + mean.abs()) * rstd
    size = q.abs().mean(dim=1, keepdim=True)
    c_off = 46 * U * size
    ch_off = 46 * U * (q * h).abs().mean(dim=1, keepdim=True) + (q.abs() * h_off).mean(dim=1, keepdim=True)
    dx_off = rstd * (c_off + h.abs() * ch_off + h_off * ch.abs() + 6 * U * (q.abs() + c.abs() + (h * ch).abs()))
    dx_off = dx_off + 2 * U * dx.abs()
    # a column: as many additions in a row as a thread has rows, at most N, sixteen threads' sums, and 64-bit ones from there
    terms = (N / 256 + 20) * U
    dw = (g * h).sum(dim=0), terms * (g * h).abs().sum(dim=0) + (g.abs() * h_off).sum(dim=0)
    db = g.sum(dim=0), terms * g.abs().sum(dim=0)
    return (dx, dx_off * (1 + half(T)) + half(T) * dx.abs() + smallest(T)), dw, db
