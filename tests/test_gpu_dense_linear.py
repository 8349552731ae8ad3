"""Dense linear layers with their epilogue (lutnn_dense_linear) and their gradients against 64-bit sums: types, sizes from one row
and one column up, strides, alignments, activations, streams, graphs.  dense_util.py derives the tolerances."""
import itertools
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


def operands(N, D, M, T, seed):
    """X with one value in 50 ten times larger, W that keeps the size, a bias, a residual, a gradient."""
    X = du.random((N, D), T, seed)
    X = torch.where(du.random((N, D), torch.float32, seed + 1) > 2.05, X * 10, X)
    return (X, du.random((D, M), T, seed + 2, D ** -0.5), du.random((M,), torch.float32, seed + 3, 0.1), du.random((N, M), T, seed + 4),
            du.random((N, M), T, seed + 5))


# rows, inputs, outputs: single ones, one less and one more than tiles and vectors, long sums with few outputs
SIZES = [(1, 1, 1), (1, 768, 768), (2, 8, 8), (3, 5, 7), (4, 1000, 264), (7, 129, 65), (8, 4096, 72), (9, 64, 200), (16, 520, 1032),
         (17, 33, 31), (33, 256, 128), (63, 515, 130), (64, 64, 64), (65, 65, 65), (100, 2048, 96), (128, 72, 512), (129, 127, 257),
         (130, 768, 768), (200, 40, 1000), (255, 260, 255), (256, 512, 256), (257, 96, 384), (300, 16, 8), (513, 1, 64), (700, 300, 1),
         (1000, 264, 520), (1025, 1030, 515)]


@pytest.mark.parametrize("kind", list(du.TYPES))
@pytest.mark.parametrize("N,D,M", SIZES)
def test_forward(lut, N, D, M, kind):
    X, W, b, R, _ = operands(N, D, M, du.TYPES[kind], seed=N + D + M)
    for i, activation in enumerate(du.ACTIVATIONS):
        bias, residual = (b, None)[i % 2], (None, R, R)[i % 3]
        Z = torch.full_like(R, float("nan")) if i in (0, 2, 3) else None
        Y = lut.dense_linear(X, W, bias, activation, residual, preactivation=Z)
        y, y_off, z, z_off = du.dense64(X, W, bias, activation, residual)
        du.check(Y, y, y_off)
        if Z is not None:
            du.check(Z, z, z_off)


@pytest.mark.parametrize("kind", list(du.TYPES))
@pytest.mark.parametrize("N,D,M", SIZES)
def test_backward(lut, N, D, M, kind):
    T = du.TYPES[kind]
    X, W, _, _, G = operands(N, D, M, T, seed=N + D + M)
    Z = du.random((N, M), T, seed=5, scale=2)
    for activation in du.ACTIVATIONS:
        got = lut.dense_linear_backward(X, W, G, Z if activation else None, activation)
        for g, (want, off) in zip(got, du.dense_backward64(X, W, G, Z, activation)):
            du.check(g, want, off)


# sizes that fill the chip with the large tiles, leave a few tiles over, and have long sums with few outputs
LARGE = [(4096, 768, 2304), (2000, 640, 640), (513, 2048, 1032), (64, 4096, 512), (8192, 264, 4096), (1000, 4104, 264), (8200, 2056, 2040),
         (4099, 1000, 1800)]


@pytest.mark.parametrize("kind", list(du.TYPES))
@pytest.mark.parametrize("N,D,M", LARGE)
def test_large(lut, N, D, M, kind):
    T = du.TYPES[kind]
    X, W, b, R, G = operands(N, D, M, T, seed=N + D + M)
    for activation, residual, keep in (("gelu", None, True), (None, R, False), ("silu", R, False)):
        Z = torch.full_like(R, float("nan")) if keep else None
        Y = lut.dense_linear(X, W, b, activation, residual, preactivation=Z)
        y, y_off, z, z_off = du.dense64(X, W, b, activation, residual)
        du.check(Y, y, y_off)
        if keep:
            du.check(Z, z, z_off)
    for activation in (None, "gelu_tanh"):
        wanted = du.dense_backward64(X, W, G, R, activation)
        for needs in ((True, True, True), (True, False, False), (False, True, True)):
            got = lut.dense_linear_backward(X, W, G, R if activation else None, activation, *needs)
            for g, (want, off) in zip(got, wanted):
                if g is not None:
                    du.check(g, want, off)


@pytest.mark.parametrize("kind", list(du.TYPES))
@pytest.mark.parametrize("N", [1, 511, 2047, 2048, 2049])
def test_bias_gradient_with_and_without_a_pass_of_its_own(lut, N, kind):
    T = du.TYPES[kind]
    for D, M, pad in ((24, 40, 8), (24, 40, 3), (520, 33, 0), (64, 1000, 24)):
        X, W, _, _, G = operands(N, D, M, T, seed=N + D)
        given = du.strided(G, pad, 8)
        got = lut.dense_linear_backward(X, W, given)
        for g, (want, off) in zip(got, du.dense_backward64(X, W, G, None, None)):
            du.check(g, want, off)
        assert torch.equal(got[2], lut.dense_linear_backward(X, W, given)[2])


@pytest.mark.parametrize("kind", list(du.TYPES))
@pytest.mark.parametrize("N", [1, 2, 3, 4, 5, 7, 8, 9])
def test_few_rows(lut, N, kind):
    """Of small and of large W, of widths that are whole strips of columns and that are not."""
    for D, M, pad in ((130, 4096, 0), (2050, 4100, 3), (1024, 8192, 8), (1030, 8203, 1), (300, 17, 0), (4097, 1021, 2), (2048, 40, 0)):
        X, W, b, R, _ = operands(N, D, M, du.TYPES[kind], seed=N + D)
        if pad:
            X, W, R = (du.strided(t, pad) for t in (X, W, R))
        Y = lut.dense_linear(X, W, b, "silu", R)
        du.check(Y, *du.dense64(X, W, b, "silu", R)[:2])


# some hundred rows, and more of odd widths: tiles that end early on either side and in k, widths around a load's four or eight values
MIDDLE = [(300, 65, 67), (1000, 100, 300), (257, 129, 5), (500, 5, 129), (700, 4, 4), (600, 3, 900), (600, 900, 3), (65, 1000, 1001),
          (2000, 33, 1), (90, 4100, 260), (2050, 1001, 1003), (4099, 1003, 1801), (200, 9, 15), (300, 7, 500), (300, 500, 7), (513, 127, 8)]


@pytest.mark.parametrize("kind", list(du.TYPES))
@pytest.mark.parametrize("pad", [0, 1])
@pytest.mark.parametrize("N,D,M", MIDDLE)
def test_middle_sizes(lut, N, D, M, pad, kind):
    X, W, b, R, G = operands(N, D, M, du.TYPES[kind], seed=N + D + M)
    if pad:
        X, W, R, G = (du.strided(t, pad, 1) for t in (X, W, R, G))
    Y = lut.dense_linear(X, W, b, "gelu", R)
    du.check(Y, *du.dense64(X, W, b, "gelu", R)[:2])
    for activation in (None, "gelu"):
        wanted = du.dense_backward64(X, W, G, R, activation)
        for needs in ((True, True, True), (True, False, False), (False, True, False)):
            got = lut.dense_linear_backward(X, W, G, R if activation else None, activation, *needs)
            for g, (want, off) in zip(got, wanted):
                if g is not None:
                    du.check(g, want, off)


@pytest.mark.parametrize("needs", list(itertools.product((False, True), repeat=3)))
def test_what_is_not_needed_changes_nothing(lut, needs):
    X, W, _, _, G = operands(70, 136, 72, torch.bfloat16, seed=3)
    Z = du.random((70, 72), torch.bfloat16, seed=6)
    whole = lut.dense_linear_backward(X, W, G, Z, "gelu")
    part = lut.dense_linear_backward(X, W, G, Z, "gelu", *needs)
    for needed, a, b in zip(needs, part, whole):
        assert torch.equal(a, b) if needed else a is None


@pytest.mark.parametrize("kind", list(du.TYPES))
@pytest.mark.parametrize("pad,shift", [(0, 1), (1, 0), (3, 5), (8, 0), (8, 8), (64, 2)])
def test_strides_and_alignment(lut, kind, pad, shift):
    """Rows that start anywhere give what dense ones give, and nothing between the rows is written."""
    T = du.TYPES[kind]
    for N, D, M in ((5, 96, 72), (150, 264, 200)):
        X, W, b, R, G = operands(N, D, M, T, seed=11)
        x, w, r, g = (du.strided(t, pad, shift) for t in (X, W, R, G))
        out, Z = du.strided(torch.zeros_like(R), pad, shift), du.strided(torch.zeros_like(R), pad, shift)
        y, y_off, z, z_off = du.dense64(X, W, b, "gelu", R)
        assert lut.dense_linear(x, w, b, "gelu", r, out=out, preactivation=Z) is out
        du.check(out, y, y_off)
        du.check(Z, z, z_off)
        if pad:
            for t in (out, Z):
                whole = torch.as_strided(t, (N, M + pad), (M + pad, 1), t.storage_offset())
                assert torch.isnan(whole[:, M:]).all()
        for got, (want, off) in zip(lut.dense_linear_backward(x, w, g, Z, "gelu"), du.dense_backward64(X, W, G, Z, "gelu")):
            du.check(got, want, off)


def test_a_single_row_has_no_stride(lut):
    X, W, b, R, G = operands(1, 40, 24, torch.float32, seed=2)
    odd = torch.as_strided(X, (1, 40), (7, 1))
    assert torch.equal(lut.dense_linear(odd, W, b), lut.dense_linear(X, W, b))


@pytest.mark.parametrize("kind", list(du.TYPES))
def test_no_rows(lut, kind):
    X, W, b, R, G = operands(4, 24, 16, du.TYPES[kind], seed=2)
    assert lut.dense_linear(X[:0], W, b, "gelu", R[:0], preactivation=R[:0].clone()).shape == (0, 16)
    dX, dW, db = lut.dense_linear_backward(X[:0], W, G[:0], R[:0], "gelu")
    assert dX.shape == (0, 24) and not dW.any() and not db.any() and dW.shape == W.shape


@pytest.mark.parametrize("kind", list(du.TYPES))
def test_values_that_are_not_finite_stay_where_they_belong(lut, kind):
    """An infinite or missing value reaches its row (of X) or its column (of W) alone, as what the sums make of it."""
    T = du.TYPES[kind]
    for N, M in ((6, 72), (150, 72), (2500, 640)):
        X, W, b, R, G = operands(N, 136, M, T, seed=21)
        X[2, 7], X[4, 130] = float("inf"), float("nan")
        W[5, 11] = float("-inf")
        with_inf = X.float() @ W.float() + b
        got = lut.dense_linear(X, W, b).float()
        assert torch.isnan(got).equal(torch.isnan(with_inf))
        assert torch.isinf(got).equal(torch.isinf(with_inf))
        whole = torch.isinf(got)
        assert torch.equal(got[whole], with_inf[whole])
        dX, dW, db = lut.dense_linear_backward(X, W, G)
        for g, want in ((dX, G.float() @ W.float().t()), (dW, X.float().t() @ G.float())):
            assert torch.isnan(g).equal(torch.isnan(want)) and torch.isinf(g).equal(torch.isinf(want))


@pytest.mark.parametrize("kind", list(du.TYPES))
@pytest.mark.parametrize("N", [3, 40, 700])
def test_activations_far_from_zero(lut, N, kind):
    """Infinite, missing and very large preactivations, on the way there and back."""
    T = du.TYPES[kind]
    far = [float("inf"), float("nan"), 6e4, 110.0, 31.0, 6.0, -6.0, -31.0, -110.0, -6e4] + ([1e30, -1e30] if kind != "f16" else [])
    X = torch.tensor((far * N)[:N * 4], dtype=T, device="cuda").view(-1, 1)
    W = torch.ones((1, 8), dtype=T, device="cuda")
    wide = X.expand(-1, 8).contiguous()
    G = torch.ones_like(wide)
    minus = wide.clone()
    minus[torch.isposinf(minus)] = float("-inf")
    for activation in du.ACTIVATIONS[1:]:
        Y, want = lut.dense_linear(X, W, None, activation), du.act64(wide.double(), activation)
        assert torch.isnan(Y).equal(torch.isnan(want)) and torch.isinf(Y).equal(torch.isinf(want.to(T)))
        fine = torch.isfinite(want.to(T))
        du.check(Y[fine], want[fine], 2.0 ** -20 * (want[fine].abs() + 1) + du.half(T) * want[fine].abs() + du.smallest(T))
        for Z in (wide, minus):
            db = lut.dense_linear_backward(X, W, G, Z, activation)[2]
            assert torch.isnan(db).all() == bool(activation != "relu" and torch.isnan(Z).any())
            some = ~torch.isnan(Z[:, 0])
            _, _, db = lut.dense_linear_backward(X[some], W, G[some], Z[some], activation)
            limits = torch.where(torch.isinf(Z), (Z > 0).double(), du.slope64(Z.double().clamp(-1e4, 1e4), activation))[some]
            du.check(db, limits.sum(0), 2.0 ** -18 * limits.abs().sum(0) + 2.0 ** -20 * len(limits))


def test_fp32_values_of_any_size(lut):
    """Very large and very small operands keep the precision of fp32 products."""
    for exponent in (-50, -30, 30, 50):
        for N in (3, 140, 2100):
            X, W, _, _, G = operands(N, 200, 520, torch.float32, seed=8)
            X, W = X * 2.0 ** exponent, W * 2.0 ** (exponent // 2)
            y, y_off, _, _ = du.dense64(X, W)
            du.check(lut.dense_linear(X, W), y, y_off)
            for g, (want, off) in zip(lut.dense_linear_backward(X, W, G), du.dense_backward64(X, W, G, None, None)):
                du.check(g, want, off)


@pytest.mark.parametrize("kind", list(du.TYPES))
def test_calls_repeat_bit_for_bit_and_in_other_streams(lut, kind):
    X, W, b, R, G = operands(300, 520, 264, du.TYPES[kind], seed=4)
    first = lut.dense_linear(X, W, b, "silu", R), *lut.dense_linear_backward(X, W, G, R, "silu")
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    results = []
    for stream in streams:  # two calls at once, each with its own workspace
        with torch.cuda.stream(stream):
            results.append((lut.dense_linear(X, W, b, "silu", R), *lut.dense_linear_backward(X, W, G, R, "silu")))
    torch.cuda.synchronize()
    for result in results:
        for a, c in zip(first, result):
            assert torch.equal(a, c)


@pytest.mark.parametrize("kind", list(du.TYPES))
@pytest.mark.parametrize("N", (1, 7, 200))
def test_captured(lut, N, kind):
    """Forward and backward in one graph: every replay, on new inputs and with eager work between, gives the eager result."""
    T = du.TYPES[kind]
    X, W, b, R, G = operands(N, 264, 520, T, seed=9)
    Z = torch.empty_like(R)

    def step():
        return (lut.dense_linear(X, W, b, "gelu", R, preactivation=Z), Z, *lut.dense_linear_backward(X, W, G, Z, "gelu"))

    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        step()
    torch.cuda.current_stream().wait_stream(stream)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = step()
    for seed in (31, 32, 33):
        for t, n in zip((X, W, b, R, G), operands(N, 264, 520, T, seed)):
            t.copy_(n)
        graph.replay()
        torch.cuda.synchronize()
        held = [t.clone() for t in captured]
        for a, c in zip(held, step()):
            assert torch.equal(a, c)


def test_long_rows_and_many_outputs(lut):
    """Offsets past 32 bits: an output of more than 2^31 bytes, and an operand whose rows lie 2^31 bytes apart."""
    N, D, M = 70000, 24, 16400
    X, W = du.random((N, D), torch.bfloat16, 1), du.random((D, M), torch.bfloat16, 2)
    Y = lut.dense_linear(X, W)
    for rows in (slice(0, 3), slice(65500, 65560), slice(N - 3, N)):
        y, off, _, _ = du.dense64(X[rows], W)
        du.check(Y[rows], y, off)
    del Y
    memory = torch.empty((1 << 30) * 2 + 64, dtype=torch.bfloat16, device="cuda")
    far = torch.as_strided(memory, (3, 24), (1 << 30, 1))
    far.copy_(X[:3])
    y, off, _, _ = du.dense64(X[:3], W)
    du.check(lut.dense_linear(far, W), y, off)


@pytest.mark.parametrize("kind", ["f32", "bf16"])
def test_many_narrow_rows(lut, kind):
    """More blocks of 16 rows than a launch has workgroups.  dW and dbias are whole numbers that fp32 holds in any order."""
    N, T = (1 << 25) + 77, du.TYPES[kind]
    X = torch.zeros((N, 3), dtype=T, device="cuda")
    X[::16] = 1
    X[-1] = 1
    W = torch.tensor([[1, 2], [3, 4], [5, 6]], dtype=T, device="cuda")
    Y = lut.dense_linear(X, W, torch.ones(2, device="cuda"))
    assert torch.equal(Y, X[:, :1] * torch.tensor([9, 12], dtype=T, device="cuda") + 1)
    G = torch.ones((N, 2), dtype=T, device="cuda")
    G[1::2] = 0
    G[-2:] = 1
    dX, dW, db = lut.dense_linear_backward(X, W, G)
    assert torch.equal(dX, G[:, :1] * torch.tensor([3, 7, 11], dtype=T, device="cuda"))
    count = torch.tensor(int((X[:, 0] * G[:, 0]).double().sum()), device="cuda")
    assert torch.equal(dW, count.to(T).expand(3, 2)) and db.eq(float(G[:, 0].double().sum())).all()


@pytest.mark.parametrize("kind", list(du.TYPES))
def test_module_gradients(lut, kind):
    """The module's gradients are the call's; fp32 ones are also those of differences."""
    from paper_2302_03213_amd.dense import DenseLinear
    T = du.TYPES[kind]
    X, W, b, R, G = operands(33, 40, 24, T, seed=14)
    layer = DenseLinear(W, b, "gelu")
    x, r = X.clone().requires_grad_(), R.clone().requires_grad_()
    Y = layer(x, r)
    Y.backward(G.t().contiguous().t())  # a gradient whose rows are not contiguous
    Z = torch.empty_like(R)
    assert torch.equal(Y, lut.dense_linear(X, W, b, "gelu", R, preactivation=Z))
    dX, dW, db = lut.dense_linear_backward(X, W, G, Z, "gelu")
    assert torch.equal(x.grad, dX) and torch.equal(layer.W.grad, dW) and torch.equal(layer.bias.grad, db) and torch.equal(r.grad, G)
    if T != torch.float32:
        return
    # central differences of the 64-bit operator along a random direction; the gradients' own errors are of fp32
    dx, dw, dv = (du.random(t.shape, torch.float32, 40 + i).double() for i, t in enumerate((X, W, b)))
    h = 1e-5

    def loss(s):
        return (du.dense64(X.double() + s * dx, W.double() + s * dw, b.double() + s * dv, "gelu")[0] * G.double()).sum()

    along = (dX.double() * dx).sum() + (dW.double() * dw).sum() + (db.double() * dv).sum()
    # h^2 of the third derivative (each of N M terms below 1, weighed by G), and 64-bit cancellation over 2 h; fp32 gradients
    size = (dX.double() * dx).abs().sum() + (dW.double() * dw).abs().sum() + (db.double() * dv).abs().sum()
    assert abs((loss(h) - loss(-h)) / (2 * h) - along) <= 1e-5 * size


def test_module_without_gradients_and_partly_frozen(lut):
    from paper_2302_03213_amd.dense import DenseLinear
    X, W, b, R, G = operands(20, 24, 16, torch.bfloat16, seed=15)
    layer = DenseLinear(W, None, "relu")
    with torch.no_grad():
        assert not layer(X).requires_grad
    layer.W.requires_grad_(False)
    x = X.clone().requires_grad_()
    layer(x).sum().backward()  # an expanded gradient
    Z = lut.dense_linear(X, W)
    assert torch.equal(x.grad, lut.dense_linear_backward(X, W, torch.ones_like(Z), Z, "relu")[0]) and layer.W.grad is None


def test_module_refuses_capture(lut):
    from paper_2302_03213_amd.dense import DenseLinear
    X, W, b, R, G = operands(20, 24, 16, torch.float32, seed=16)
    layer = DenseLinear(W, b, "gelu")
    eager = layer(X)  # an eager graph of the same parameters, alive
    with pytest.raises(RuntimeError, match="cannot be captured"):
        with torch.cuda.graph(torch.cuda.CUDAGraph()):
            layer(X).backward(G)
    torch.cuda.synchronize()
    eager.backward(G)
    assert torch.isfinite(layer.W.grad).all()


@pytest.mark.parametrize("kind", list(du.TYPES))
def test_the_python_way_agrees(lut, kind, monkeypatch):
    from paper_2302_03213_amd import binding
    X, W, b, R, G = operands(70, 40, 24, du.TYPES[kind], seed=17)
    Z = torch.empty_like(R)

    def results():
        return (lut.dense_linear(X, W, b, "gelu", R, preactivation=Z), *lut.dense_linear_backward(X, W, G, R, "silu"),
                lut.dense_linear_backward(X, W, G, None, None, False, True, False)[1])

    native = results()
    monkeypatch.setattr(binding, "_calls", binding._NoCalls())
    for a, c in zip(native, results()):
        assert torch.equal(a, c)


def test_tensors_that_are_refused(lut):
    X, W, b, R, G = operands(6, 8, 16, torch.bfloat16, seed=18)
    for call in (lambda: lut.dense_linear(X, W.t()), lambda: lut.dense_linear(X, W.float()), lambda: lut.dense_linear(X, W, b[:8]),
                 lambda: lut.dense_linear(X, W, b.to(X.dtype)), lambda: lut.dense_linear(X, W, b, "swish"),
                 lambda: lut.dense_linear(X, W, residual=R[:3]), lambda: lut.dense_linear(X, W.t().contiguous().t()),
                 lambda: lut.dense_linear(X.double(), W.double()), lambda: lut.dense_linear(X, W.cpu()),
                 lambda: lut.dense_linear(X, W, out=R[:3]), lambda: lut.dense_linear_backward(X, W, G, None, "gelu"),
                 lambda: lut.dense_linear_backward(X[:5], W, G), lambda: lut.dense_linear_backward(X, W, G, G[:2], "relu")):
        with pytest.raises(ValueError):
            call()
    with pytest.raises(lut.LutnnError) as e:  # rows on top of each other
        lut.dense_linear(X[:1].expand(6, 8), W)
    assert e.value.name == "LUTNN_E_SHAPE"


def test_two_graphs_of_one_pool(lut):
    """Workspaces of two graphs may be the same memory: replayed one after the other, each gives its own result."""
    sets = [operands(N, 264, 520, torch.float32, seed=N) for N in (2200, 1500)]
    for X, W, b, R, G in sets:
        lut.dense_linear(X, W, b)
    graphs, outs, pool = [], [], None
    for X, W, b, R, G in sets:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, pool=pool):
            outs.append((lut.dense_linear(X, W, b, "gelu"), *lut.dense_linear_backward(X, W, G)))
        graphs.append(graph)
        pool = graph.pool()
    wanted = [(lut.dense_linear(X, W, b, "gelu"), *lut.dense_linear_backward(X, W, G)) for X, W, b, R, G in sets]
    for i in (0, 1, 1, 0, 1):
        graphs[i].replay()
        torch.cuda.synchronize()
        for a, c in zip(outs[i], wanted[i]):
            assert torch.equal(a, c)
