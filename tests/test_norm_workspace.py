"""Where layer norm's gradients need a workspace, and how much.  No GPU needed: addresses are made up and never dereferenced."""
import ctypes

import pytest

G, X, S, P = (ctypes.c_void_p(0x100000 * i) for i in range(1, 5))


@pytest.fixture(scope="module")
def lut():
    import paper_2302_03213_amd as lut_mod
    return lut_mod


@pytest.mark.parametrize("D", [32, 1025, 2048, 2049, 4096, 4097, 16384])
@pytest.mark.parametrize("N", [768, 769, 1024, 1025, 5000])
def test_what_is_asked_for(lut, N, D):
    """The query covers every type; a call refuses less than its own type needs.  (The refused calls launch nothing.)"""
    fp32_alone = 768 < N <= 1024 and 2048 < D <= 4096  # summed beside dX in 16 bits
    size = lut.LIB.lutnn_layer_norm_backward_workspace_bytes(N, D)
    assert (size > 0) == (N > 1024 or fp32_alone)
    assert size % (2 * D * 4) == 0
    for dtype in (0, 1, 2) if N > 1024 else (0,) if fp32_alone else ():
        for workspace, given, status in ((None, size, "LUTNN_E_NULL"), (P, size - 1, "LUTNN_E_SHAPE")):
            got = lut.LIB.lutnn_layer_norm_backward(dtype, G, N, D, X, D, D, S, None, None, 0, None, 0, P, P, workspace, given, None)
            assert lut.LIB.lutnn_status_string(got).decode() == status


def test_rows_that_pass_the_cache(lut):
    """One workgroup per compute unit leaves half the sums; the room is for two where a type may take them."""
    with lut.tunables(LUTNN_NORM_SUMS="1"):
        one = lut.LIB.lutnn_layer_norm_backward_workspace_bytes(16384, 4096)
    assert lut.LIB.lutnn_layer_norm_backward_workspace_bytes(16384, 4096) == 2 * one
