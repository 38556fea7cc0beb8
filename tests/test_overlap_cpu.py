"""Overlapping memory is refused by the operators between the quantized layers before anything is launched."""
import ctypes as C

import pytest

from paper_2510_02822_b200 import binding as fx
from paper_2510_02822_b200 import build as fxbuild


@pytest.fixture(scope="module")
def lib():
    fxbuild.build_library()
    return fx.lib()


X = 1 << 20      # never dereferenced


def call(lib, y, x_dtype, y_dtype, Nb=3, P=5, channels=32):
    return lib.flexiq_group_norm(C.c_void_p(X), x_dtype, Nb, P, channels, 4, None, None, 1e-5, 0, y_dtype, C.c_void_p(y), None, None)


@pytest.mark.parametrize("x_dtype, y_dtype", [(0, 0), (1, 1), (2, 0), (0, 2)])
def test_group_norm(lib, x_dtype, y_dtype):
    size = {0: 4, 1: 2, 2: 2}
    n = 3 * 5 * 32
    for y in (X + 16, X - 16, X + n * size[x_dtype] - 16, X - n * size[y_dtype] + 16):
        assert call(lib, y, x_dtype, y_dtype) == fx.ERR_INVALID_ARG
        assert "overlap" in fx.last_error()
    # side by side, and nothing at all, are no overlaps: what is refused then, if anything, is the machine without a GPU
    for y in (X + n * size[x_dtype], X - n * size[y_dtype]):
        if call(lib, y, x_dtype, y_dtype, Nb=0) != fx.OK:
            assert "overlap" not in fx.last_error()
    assert call(lib, X + 16, x_dtype, y_dtype, Nb=0) == fx.OK
