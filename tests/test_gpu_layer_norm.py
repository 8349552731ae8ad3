"""Layer norm (lutnn_layer_norm) and its gradients against 64-bit sums: types, widths from one value up, strides, residuals, rows
without spread, streams, graphs.  dense_util.py derives the tolerances."""
import itertools
import sys

import pytest
import torch

import dense_util as du

pytestmark = pytest.mark.gpu

EPS = 1e-5


@pytest.fixture(scope="module")
def lut():
    import paper_2302_03213_amd as lut_mod
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    return lut_mod


@pytest.fixture(autouse=True)
def announce(request):
    print("\n[case] %s" % request.node.nodeid, file=sys.stderr, flush=True)
    yield


def operands(N, D, T, seed, shift=0.0):
    X, R, G = (du.random((N, D), T, seed + i) for i in range(3))
    return X + shift, R, G, 1 + du.random((D,), torch.float32, seed + 3, 0.1), du.random((D,), torch.float32, seed + 4, 0.1)


# widths around vectors, wavefronts and the steps of the threads per row
SIZES = [(1, 1), (3, 2), (5, 3), (4, 7), (9, 8), (17, 9), (33, 63), (2, 64), (40, 65), (16, 255), (31, 256), (33, 257), (1, 768),
         (130, 768), (7, 1000), (5, 1023), (6, 1024), (6, 1025), (3, 2049), (600, 1536), (2, 4095), (3, 4096), (3, 4097), (2, 9000), (3, 8192), (4, 5120),
                  (2, 16383), (3, 16384), (5000, 40), (2100, 264)]


@pytest.mark.parametrize("kind", list(du.TYPES))
@pytest.mark.parametrize("N,D", SIZES)
def test_forward(lut, N, D, kind):
    X, R, _, w, b = operands(N, D, du.TYPES[kind], seed=N + D)
    for residual, weight, bias in ((None, w, b), (R, w, b), (R, None, None), (None, w, None), (None, None, b)):
        total = torch.full_like(X, float("nan")) if residual is not None else None
        statistics = torch.full((N, 2), float("nan"), device="cuda")
        Y = lut.layer_norm(X, weight, bias, EPS, residual, total=total, statistics=statistics)
        y, s, mean, rstd = du.norm64(X, weight, bias, EPS, residual)
        du.check(Y, *y)
        du.check(statistics[:, :1], *mean)
        du.check(statistics[:, 1:], *rstd)
        if total is not None:
            du.check(total, *s)
        assert torch.equal(Y, lut.layer_norm(X, weight, bias, EPS, residual))


@pytest.mark.parametrize("kind", list(du.TYPES))
@pytest.mark.parametrize("N,D", SIZES)
def test_backward(lut, N, D, kind):
    X, R, G, w, b = operands(N, D, du.TYPES[kind], seed=N + D)
    statistics = torch.empty((N, 2), device="cuda")
    lut.layer_norm(X, statistics=statistics)
    for weight, residual in ((w, None), (w, R), (None, None)):
        got = lut.layer_norm_backward(G, X, statistics, weight, residual)
        for g, want in zip(got, du.norm_backward64(G, X, statistics, weight, residual)):
            du.check(g, *want)


@pytest.mark.parametrize("needs", list(itertools.product((False, True), repeat=3)))
def test_what_is_not_needed_changes_nothing(lut, needs):
    X, R, G, w, b = operands(70, 136, torch.bfloat16, seed=3)
    statistics = torch.empty((70, 2), device="cuda")
    lut.layer_norm(X, statistics=statistics)
    whole = lut.layer_norm_backward(G, X, statistics, w, R)
    part = lut.layer_norm_backward(G, X, statistics, w, R, *needs)
    for needed, a, c in zip(needs, part, whole):
        assert torch.equal(a, c) if needed else a is None


@pytest.mark.parametrize("kind", list(du.TYPES))
@pytest.mark.parametrize("pad,shift", [(0, 1), (1, 0), (3, 5), (8, 0), (64, 2)])
def test_strides_and_alignment(lut, kind, pad, shift):
    for N, D in ((5, 200), (70, 1001)):
        X, R, G, w, b = operands(N, D, du.TYPES[kind], seed=6)
        x, r, g = (du.strided(t, pad, shift) for t in (X, R, G))
        out, total = (du.strided(torch.zeros_like(X), pad, shift) for _ in range(2))
        statistics = torch.empty((N, 2), device="cuda")
        plain_total, plain_statistics = torch.empty_like(X), torch.empty((N, 2), device="cuda")
        want = lut.layer_norm(X, w, b, EPS, R, total=plain_total, statistics=plain_statistics)
        assert torch.equal(lut.layer_norm(x, w, b, EPS, r, out=out, total=total, statistics=statistics), want)
        assert torch.equal(total, plain_total) and torch.equal(statistics, plain_statistics)
        if pad:
            for t in (out, total):
                assert torch.isnan(torch.as_strided(t, (N, D + pad), (D + pad, 1), t.storage_offset())[:, D:]).all()
        for a, c in zip(lut.layer_norm_backward(g, total, statistics, w, r), lut.layer_norm_backward(G, plain_total, statistics, w, R)):
            assert torch.equal(a, c)


@pytest.mark.parametrize("kind", list(du.TYPES))
def test_rows_without_spread_and_far_from_zero(lut, kind):
    """Constant rows give the bias; a common shift of a row, large against its spread, costs what the shift's own steps cost."""
    T = du.TYPES[kind]
    for D in (1, 100, 768, 3000):
        X = torch.full((4, D), 3.5, dtype=T, device="cuda")
        X[1:3] = 0
        b = du.random((D,), torch.float32, 2)
        y, _, _, _ = du.norm64(X, None, b, EPS, None)
        du.check(lut.layer_norm(X, None, b, EPS), *y)
        X, _, _, w, b = operands(6, D, T, seed=8, shift=100.0)
        y, _, _, _ = du.norm64(X, w, b, EPS, None)
        du.check(lut.layer_norm(X, w, b, EPS), *y)


@pytest.mark.parametrize("kind", list(du.TYPES))
def test_a_row_that_is_not_finite_is_alone(lut, kind):
    X, R, G, w, b = operands(40, 264, du.TYPES[kind], seed=9)
    statistics = torch.empty((40, 2), device="cuda")
    want = lut.layer_norm(X, w, b, EPS, statistics=statistics)
    dX = lut.layer_norm_backward(G, X, statistics, w)[0]
    X[7, 100], X[21, 0] = float("inf"), float("nan")
    got = lut.layer_norm(X, w, b, EPS, statistics=statistics)
    back = lut.layer_norm_backward(G, X, statistics, w)[0]
    others = [n for n in range(40) if n not in (7, 21)]
    assert torch.equal(got[others], want[others]) and torch.equal(back[others], dX[others])
    assert torch.isnan(got[[7, 21]]).all()


@pytest.mark.parametrize("kind", list(du.TYPES))
def test_no_rows(lut, kind):
    X, R, G, w, b = operands(3, 40, du.TYPES[kind], seed=2)
    statistics = torch.empty((0, 2), device="cuda")
    assert lut.layer_norm(X[:0], w, b, EPS, R[:0], total=R[:0].clone(), statistics=statistics).shape == (0, 40)
    dX, dw, db = lut.layer_norm_backward(G[:0], X[:0], statistics, w)
    assert dX.shape == (0, 40) and not dw.any() and not db.any() and dw.shape == (40,)


def test_offsets_past_32_bits(lut):
    N, D = 140000, 16384
    X = torch.empty((N, D), dtype=torch.bfloat16, device="cuda")
    small = du.random((16, D), torch.bfloat16, 1)
    for at in (0, N // 2, N - 16):
        X[at:at + 16] = small
    X[16:N // 2] = 0
    X[N // 2 + 16:N - 16] = 0
    Y = lut.layer_norm(X)
    y, _, _, _ = du.norm64(small, None, None, EPS, None)
    for at in (0, N // 2, N - 16):
        du.check(Y[at:at + 16], *y)


@pytest.mark.parametrize("D", [1, 5])
def test_more_rows_than_a_launch_has_workgroups_for(lut, D):
    N = (1 << 25) + 33  # 2^21 workgroups of 16 rows, and some
    X = torch.zeros((N, D), dtype=torch.bfloat16, device="cuda")
    small = du.random((40, D), torch.bfloat16, D)
    X[:40] = small
    X[-40:] = small
    statistics = torch.full((N, 2), float("nan"), device="cuda")
    Y = lut.layer_norm(X, eps=EPS, statistics=statistics)
    y, _, _, _ = du.norm64(small, None, None, EPS, None)
    du.check(Y[:40], *y)
    du.check(Y[-40:], *y)
    assert not Y[40:-40].any() and torch.isfinite(statistics).all()
    G = torch.ones_like(X)
    G[:-8] = 0
    dX, dw, db = lut.layer_norm_backward(G, X, statistics)
    assert db.eq(8).all() and not dX[:-8].any()
    torch.testing.assert_close(dw.double(), Y[-8:].double().sum(0), rtol=0, atol=8 * 4 * 2.0 ** -8)  # of values below 4 in bf16


@pytest.mark.parametrize("kind", list(du.TYPES))
def test_other_streams_and_repeats(lut, kind):
    X, R, G, w, b = operands(3000, 768, du.TYPES[kind], seed=4)
    statistics = torch.empty((3000, 2), device="cuda")
    first = lut.layer_norm(X, w, b, EPS, R, statistics=statistics), *lut.layer_norm_backward(G, X, statistics, w, R)
    torch.cuda.synchronize()
    results = []
    for stream in [torch.cuda.Stream() for _ in range(2)]:
        with torch.cuda.stream(stream):
            results.append((lut.layer_norm(X, w, b, EPS, R), *lut.layer_norm_backward(G, X, statistics, w, R)))
    torch.cuda.synchronize()
    for result in results:
        for a, c in zip(first, result):
            assert torch.equal(a, c)


@pytest.mark.parametrize("kind", list(du.TYPES))
@pytest.mark.parametrize("N,D", [(1, 768), (300, 264), (40, 3000)])
def test_captured(lut, N, D, kind):
    X, R, G, w, b = operands(N, D, du.TYPES[kind], seed=4)
    statistics, total = torch.empty((N, 2), device="cuda"), torch.empty_like(X)

    def step():
        Y = lut.layer_norm(X, w, b, EPS, R, total=total, statistics=statistics)
        return (Y, total, statistics, *lut.layer_norm_backward(G, total, statistics, w, G))

    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        step()
    torch.cuda.current_stream().wait_stream(stream)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = step()
    for seed in (31, 32, 33):
        for t, n in zip((X, R, G, w, b), operands(N, D, du.TYPES[kind], seed)):
            t.copy_(n)
        graph.replay()
        torch.cuda.synchronize()
        held = [t.clone() for t in captured]
        for a, c in zip(held, step()):
            assert torch.equal(a, c)


def test_module_gradients(lut):
    """The module against differences of the 64-bit operator, with the total used beside the norm, and each of them alone."""
    from paper_2302_03213_amd.dense import LayerNorm
    X, R, G, w, b = operands(12, 40, torch.float32, seed=5)
    G2 = du.random((12, 40), torch.float32, 77)
    norm = LayerNorm(40)
    with torch.no_grad():
        norm.weight.copy_(w)
        norm.bias.copy_(b)
    for use_y, use_total in ((True, True), (True, False), (False, True)):
        x, r = X.clone().requires_grad_(), R.clone().requires_grad_()
        norm.zero_grad()
        Y, total = norm(x, r, with_total=True)
        ((Y * G).sum() * use_y + (total * G2).sum() * use_total if use_y and use_total else (Y * G).sum() if use_y
         else (total * G2).sum()).backward()
        directions = [du.random(t.shape, torch.float32, 60 + i).double() for i, t in enumerate((X, R, w, b))]

        def loss(h):
            s = X.double() + R.double() + h * (directions[0] + directions[1])
            y = torch.nn.functional.layer_norm(s, (40,), w.double() + h * directions[2], b.double() + h * directions[3], EPS)
            return (y * G.double()).sum() * use_y + (s * G2.double()).sum() * use_total

        grads = [x.grad, r.grad, norm.weight.grad, norm.bias.grad]
        parts = [(g.double() * d) for g, d in zip(grads, directions) if g is not None]
        along, size = sum(p.sum() for p in parts), sum(p.abs().sum() for p in parts)
        # h^2 of third derivatives of order one, 64-bit cancellation over 2 h, fp32 gradients
        assert abs((loss(1e-5) - loss(-1e-5)) / 2e-5 - along) <= 1e-5 * size


def test_module_without_residual_and_refusals(lut):
    from paper_2302_03213_amd.dense import LayerNorm
    X, _, G, _, _ = operands(12, 40, torch.bfloat16, seed=5)
    norm = LayerNorm(40)
    x = X.clone().requires_grad_()
    Y = norm(x)
    Y.backward(G)
    statistics = torch.empty((12, 2), device="cuda")
    assert torch.equal(Y, lut.layer_norm(X, norm.weight, norm.bias, statistics=statistics))
    dX, dw, db = lut.layer_norm_backward(G, X, statistics, norm.weight)
    assert torch.equal(x.grad, dX) and torch.equal(norm.weight.grad, dw) and torch.equal(norm.bias.grad, db)
    with pytest.raises(ValueError):
        norm(X, with_total=True)
    eager = norm(X)
    with pytest.raises(RuntimeError, match="cannot be captured"):
        with torch.cuda.graph(torch.cuda.CUDAGraph()):
            norm(X).backward(G)
    torch.cuda.synchronize()
    eager.backward(G)


@pytest.mark.parametrize("kind", list(du.TYPES))
def test_the_python_way_agrees(lut, kind, monkeypatch):
    from paper_2302_03213_amd import binding
    X, R, G, w, b = operands(70, 40, du.TYPES[kind], seed=17)
    statistics, total = torch.empty((70, 2), device="cuda"), torch.empty_like(X)

    def results():
        return (lut.layer_norm(X, w, b, EPS, R, total=total, statistics=statistics), total.clone(), statistics.clone(),
                *lut.layer_norm_backward(G, total, statistics, w, R))

    native = results()
    monkeypatch.setattr(binding, "_calls", binding._NoCalls())
    for a, c in zip(native, results()):
        assert torch.equal(a, c)


def test_tensors_that_are_refused(lut):
    X, R, G, w, b = operands(6, 8, torch.bfloat16, seed=18)
    statistics = torch.empty((6, 2), device="cuda")
    for call in (lambda: lut.layer_norm(X, w[:4]), lambda: lut.layer_norm(X, w.to(X.dtype)), lambda: lut.layer_norm(X, w, b, residual=R[:3]),
                 lambda: lut.layer_norm(X.t()), lambda: lut.layer_norm(X.double()), lambda: lut.layer_norm(X, statistics=statistics[:3]),
                 lambda: lut.layer_norm(X, residual=R.float()), lambda: lut.layer_norm_backward(G, X, statistics.t()),
                 lambda: lut.layer_norm_backward(G, X.float(), statistics), lambda: lut.layer_norm_backward(G, X, statistics, w.cpu())):
        with pytest.raises(ValueError):
            call()
    for call in (lambda: lut.layer_norm(X, total=R), lambda: lut.layer_norm(X, eps=-1.0), lambda: lut.layer_norm(X[:1].expand(6, 8)),
                 lambda: lut.layer_norm(torch.zeros(2, 16392, device="cuda"))):
        with pytest.raises(lut.LutnnError):
            call()
