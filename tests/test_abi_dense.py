"""What the calls of the layers between the looked-up ones refuse, on the host, before anything could be launched.  No GPU needed:
the addresses are made up and never dereferenced."""
import ctypes

import pytest
import torch


@pytest.fixture(scope="module")
def lut():
    import paper_2302_03213_amd as lut_mod
    return lut_mod


class Call:
    """An entry point with arguments that it accepts, as a dict in order; refused(name=value, ...) is its status with some changed."""

    def __init__(self, lut, name, **args):
        self.lut, self.entry, self.args = lut, getattr(lut.LIB, name), args

    def refused(self, **changes):
        assert set(changes) <= set(self.args)
        values = dict(self.args, **changes)
        status = self.entry(*[ctypes.c_void_p(v) if isinstance(v, int) and v >= 0x10000 and k not in SIZES else v
                              for k, v in values.items()])
        assert status != 0 or values["N"] == 0
        return self.lut.LIB.lutnn_status_string(status).decode()


SIZES = ("N", "D", "M", "ldx", "ldw", "ldr", "ldy", "ldz", "ldg", "ldt", "lddx", "lddw", "bytes")


def forward(lut):
    return Call(lut, "lutnn_dense_linear", dtype=1, X=0x10000, N=64, ldx=32, W=0x20000, ldw=16, D=32, M=16, bias=0x30000, act=2,
                R=0x40000, ldr=16, Y=0x50000, ldy=16, Z=0x60000, ldz=16, workspace=0x70000, bytes=1 << 40, stream=None)


def backward(lut):
    return Call(lut, "lutnn_dense_linear_backward", dtype=1, X=0x10000, N=64, ldx=32, W=0x20000, ldw=16, D=32, M=16, G=0x30000, ldg=16,
                Z=0x40000, ldz=16, act=2, dX=0x50000, lddx=32, dW=0x60000, lddw=16, db=0x70000, workspace=0x80000, bytes=1 << 40,
                stream=None)


def norm(lut):
    return Call(lut, "lutnn_layer_norm", dtype=1, X=0x10000, N=64, ldx=32, D=32, R=0x20000, ldr=32, w=0x30000, b=0x40000, eps=1e-5,
                Y=0x50000, ldy=32, S=0x60000, ldt=32, statistics=0x70000, stream=None)


def norm_backward(lut):
    return Call(lut, "lutnn_layer_norm_backward", dtype=1, G=0x10000, N=64, ldg=32, X=0x20000, ldx=32, D=32, statistics=0x30000,
                w=0x40000, R=0x50000, ldr=32, dX=0x60000, lddx=32, dw=0x70000, db=0x80000, workspace=0x90000, bytes=1 << 40,
                stream=None)


@pytest.mark.parametrize("make", [forward, backward, norm, norm_backward])
def test_refusals_common_to_all(lut, make):
    call = make(lut)
    for dtype in (-1, 3):
        assert call.refused(dtype=dtype) == "LUTNN_E_UNSUPPORTED"
    assert call.refused(N=-1) == "LUTNN_E_SHAPE" and call.refused(N=1 << 31) == "LUTNN_E_SHAPE"
    assert call.refused(D=0) == "LUTNN_E_SHAPE" and call.refused(D=-4) == "LUTNN_E_SHAPE"
    assert call.refused(D=1 << 30) in ("LUTNN_E_SHAPE", "LUTNN_E_UNSUPPORTED")
    for name in call.args:
        if name.startswith("ld"):
            assert call.refused(**{name: 15}) == "LUTNN_E_SHAPE", name
            assert call.refused(**{name: (1 << 32) + 1}) == "LUTNN_E_SHAPE", name
    for name in ("X", "W", "G", "R", "Y", "Z", "S", "dX", "dW"):
        if name in call.args:
            assert call.refused(**{name: call.args[name] + 1}) == "LUTNN_E_ALIGN", name
            assert call.refused(dtype=0, **{name: call.args[name] + 2}) == "LUTNN_E_ALIGN", name
    for name in ("bias", "w", "b", "db", "dw", "statistics"):
        if name in call.args:
            assert call.refused(**{name: call.args[name] + 2}) == "LUTNN_E_ALIGN", name


def test_dense_linear_refusals(lut):
    call = forward(lut)
    for name in ("X", "W", "Y"):
        assert call.refused(**{name: None}) == "LUTNN_E_NULL", name
    for act in (-1, 5):
        assert call.refused(act=act) == "LUTNN_E_UNSUPPORTED"
    assert call.refused(M=0) == "LUTNN_E_SHAPE" and call.refused(M=(1 << 21) + 1, ldw=1 << 22, ldr=1 << 22, ldy=1 << 22, ldz=1 << 22) == "LUTNN_E_SHAPE"
    assert call.refused(N=0, X=None, W=None, Y=None, workspace=None) == "LUTNN_OK"
    assert call.refused(N=(1 << 28) + 1) == "LUTNN_E_SHAPE"  # 2^21 tiles of 128 rows
    assert call.refused(N=(1 << 27) + 1, M=257, ldw=264, ldr=264, ldy=264, ldz=264) == "LUTNN_E_SHAPE"


def test_dense_linear_backward_refusals(lut):
    call = backward(lut)
    for name in ("X", "W", "G", "Z", "workspace"):
        assert call.refused(**{name: None}) == "LUTNN_E_NULL", name
    assert call.refused(act=9) == "LUTNN_E_UNSUPPORTED"
    assert call.refused(workspace=0x80004) == "LUTNN_E_ALIGN"
    assert call.refused(bytes=15) == "LUTNN_E_SHAPE"


def test_layer_norm_refusals(lut):
    call = norm(lut)
    for name in ("X", "Y", "R"):  # a total without a residual
        assert call.refused(**{name: None}) == "LUTNN_E_NULL", name
    for eps in (-1e-5, float("nan"), float("inf")):
        assert call.refused(eps=eps) == "LUTNN_E_SHAPE"
    assert call.refused(D=16385, ldx=20000) == "LUTNN_E_UNSUPPORTED"
    assert call.refused(N=0, X=None, Y=None) == "LUTNN_OK"


def test_layer_norm_backward_refusals(lut):
    call = norm_backward(lut)
    for name in ("G", "X", "statistics"):
        assert call.refused(**{name: None}) == "LUTNN_E_NULL", name
    assert call.refused(D=16385) == "LUTNN_E_UNSUPPORTED"
    assert call.refused(N=1025, workspace=None) == "LUTNN_E_NULL"  # fewer rows of that width need none
    assert call.refused(N=1025, workspace=0x90004) == "LUTNN_E_ALIGN"
    assert call.refused(N=1025, bytes=0) == "LUTNN_E_SHAPE"


def test_workspace_queries(lut):
    query, back = lut.LIB.lutnn_dense_linear_workspace_bytes, lut.LIB.lutnn_dense_linear_backward_workspace_bytes
    X, W, G, Z = (ctypes.c_void_p(0x10000 * i) for i in range(1, 5))
    for bad in ((7, X, 4, 32, W, 16, 32, 16), (1, X, 0, 32, W, 16, 32, 16), (1, X, -1, 32, W, 16, 32, 16), (1, X, 4, 31, W, 16, 32, 16),
                (1, X, 4, 32, W, 15, 32, 16), (1, X, 4, 32, W, 16, 0, 16)):
        assert query(*bad) == 0
    for bad in ((1, X, 0, 32, W, 16, 32, 16, G, 16, Z, 16, 1, 1, 1, 1), (1, X, 4, 32, W, 16, 32, 16, G, 15, Z, 16, 1, 1, 1, 1),
                (1, X, 4, 32, W, 16, 32, 16, G, 16, Z, 16, 9, 1, 1, 1), (1, X, 4, 31, W, 16, 32, 16, G, 16, Z, 16, 1, 1, 1, 1)):
        assert back(*bad) == 0
    assert lut.LIB.lutnn_layer_norm_backward_workspace_bytes(0, 40) == 0
    assert lut.LIB.lutnn_layer_norm_backward_workspace_bytes(4, 16385) == 0


def test_python_refusals(lut):
    """Tensors that are not on a GPU, of another kind or of another shape."""
    X = torch.zeros(4, 8)
    for call in (lambda: lut.dense_linear(X, torch.zeros(8, 3)), lambda: lut.dense_linear_backward(X, torch.zeros(8, 8), X),
                 lambda: lut.layer_norm(X), lambda: lut.layer_norm_backward(X, X, torch.zeros(4, 2))):
        with pytest.raises(ValueError, match="CUDA matrix"):
            call()
    from paper_2302_03213_amd import binding
    like = torch.zeros(4, 8, dtype=torch.bfloat16)
    assert binding._matrix("A", like, (4, 8), like) == 8
    assert binding._matrix("A", like[:1], (1, 8), like) == 8
    for t, shape in ((like.float(), (4, 8)), (like, (4, 7)), (torch.zeros(8, 4, dtype=torch.bfloat16).t(), (4, 8)), (like[0], (4, 8))):
        with pytest.raises(ValueError):
            binding._matrix("A", t, shape, like)
    with pytest.raises(ValueError):
        binding._activation("swish")
    for v in (torch.zeros(8), torch.zeros(7), torch.zeros(16)[::2], torch.zeros(8, dtype=torch.bfloat16), torch.zeros(1, 8)):
        good = v.dtype == torch.float32 and v.shape == (8,) and v.is_contiguous()
        if good:
            binding._vector("v", v, 8, like)
        else:
            with pytest.raises(ValueError):
                binding._vector("v", v, 8, like)


def test_native_calls_leave_alone_what_is_not_plain(lut):
    from paper_2302_03213_amd import binding
    calls, X, v = binding._calls, torch.zeros(4, 8), torch.zeros(8)
    assert calls.dense_linear(X, X, None, 0, None, None) is None
    assert calls.dense_linear(X, X, None, 0) is None
    assert calls.dense_linear_backward(X, X, X, None, 0, True, True, True) is None
    assert calls.layer_norm(X, v, v, 1e-5, None, None, None) is None
    assert calls.layer_norm_backward(X, X, X, None, None, True, True, True) is None
