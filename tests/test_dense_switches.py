"""The switches that pin a form of the dense layers' products and of layer norm's sums.  No GPU needed: addresses are made up and never
dereferenced."""
import ctypes

import pytest

import dense_forms as df

X, W, G, Z = (ctypes.c_void_p(0x100000 * i) for i in range(1, 5))


@pytest.fixture(scope="module")
def lut():
    import paper_2302_03213_amd as lut_mod
    return lut_mod


@pytest.mark.parametrize("name,good,bad", [("LUTNN_DENSE_FORM", ("few", "memory") + tuple(df.TILES), ("256", "64x32", "as is")),
                                           ("LUTNN_DENSE_SPLITS", ("1", "3", "64"), ("0", "65", "two")),
                                           ("LUTNN_NORM_SUMS", ("beside", "1", "2"), ("0", "3", "besides"))])
def test_values(lut, name, good, bad):
    try:
        for v in good:
            lut.set_tunable(name, v)
        for v in bad:
            with pytest.raises(lut.LutnnError) as e:
                lut.set_tunable(name, v)
            assert e.value.name == "LUTNN_E_SHAPE"
    finally:
        lut.set_tunable(name, None)


def laid_out(dtype, rows, width):
    return -(-(3 if dtype == 0 else 1) * rows * (-(-width // 8) * 8) * 2 // 256) * 256


def ceil(a, b):
    return -(-a // b)


@pytest.mark.parametrize("kind", list(df.FORMS))
def test_the_workspace_is_that_of_the_pinned_form(lut, kind):
    """One with shared sums has room for all of them, tile by tile; X and W laid out where the form wants that and they are not."""
    dtype, (N, D, M) = {"f32": 0, "bf16": 1, "f16": 2}[kind], (300, 264, 520)
    for form in df.FORMS[kind]:
        for splits in (1, 3):
            with lut.tunables(LUTNN_DENSE_FORM=form, LUTNN_DENSE_SPLITS=splits):
                forward = lut.LIB.lutnn_dense_linear_workspace_bytes(dtype, X, N, D, W, M, D, M)
                pair = lut.LIB.lutnn_dense_linear_backward_workspace_bytes(dtype, X, N, D, W, M, D, M, G, M, None, 0, 0, 1, 1, 0)
            if form == "memory":
                assert forward == pair == 0
                continue
            (ti, tj), as_is = df.TILES[form], form.endswith("as is")
            sums = [ceil(i, ti) * ceil(j, tj) * ti * tj * 4 * splits if splits > 1 else 0 for i, j in ((N, M), (N, D), (D, M))]
            planes = [laid_out(0, r, w) if dtype == 0 and not as_is else 0 for r, w in ((N, D), (D, M), (N, M))]
            assert forward == sums[0] + planes[0] + planes[1], (form, splits)
            assert pair == sums[1] + sums[2] + sum(planes), (form, splits)


def test_a_form_that_the_call_cannot_take_is_ignored(lut):
    def forward(dtype, N, D, M):
        return lut.LIB.lutnn_dense_linear_workspace_bytes(dtype, X, N, D, W, M, D, M)

    for dtype, form, size in ((0, "256x256", (300, 264, 520)), (1, "memory", (300, 264, 520)), (1, "few", (300, 264, 520)),
                              (1, "64x64 as is", (300, 264, 5)), (0, "32x32 as is", (300, 264, 3))):
        free = forward(dtype, *size)
        with lut.tunables(LUTNN_DENSE_FORM=form):
            assert forward(dtype, *size) == free, (dtype, form)
    free = forward(1, 300, 64, 520)
    with lut.tunables(LUTNN_DENSE_SPLITS=64):  # more than a sum of 64 has stages
        assert forward(1, 300, 64, 520) == free


def test_norm_sums(lut):
    query = lut.LIB.lutnn_layer_norm_backward_workspace_bytes
    with lut.tunables(LUTNN_NORM_SUMS="beside"):
        assert query(5000, 2000) == 0
    with lut.tunables(LUTNN_NORM_SUMS="1"):
        one = query(5000, 2000)
        assert query(100, 2000) == 100 * 2 * 2000 * 4  # as many workgroups as rows
    with lut.tunables(LUTNN_NORM_SUMS="2"):
        assert query(5000, 2000) == 2 * one > 0
