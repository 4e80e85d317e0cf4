"""The experts' MLP entry points at and past the ends of their sizes, on the host (no GPU needed: the
pointers are never followed)."""
import ctypes

import pytest

from .test_mlp_abi import SHAPE, _mx, _refuse, lib  # noqa: F401 (lib: a fixture)


@pytest.mark.parametrize("batch,rows,cols", [
    ((1 << 31) - 1, 1 << 40, 64), ((1 << 31) - 1, 1 << 33, 32), ((1 << 31) - 1, (1 << 40) - 1, 1 << 24),
    (1 << 20, 1 << 39, 1 << 25), (2, (1 << 34) + 1, 32), (1, (1 << 35) + 1, 32)])
def test_quantize_sizes_whose_product_passes_64_bits(lib, batch, rows, cols):  # noqa: F811
    """More than 2^40 elements, also where their count overflows 64 bits."""
    # (no x: a check that let the sizes pass would launch nothing)
    change = dict(x=None, batch=batch, rows=rows, cols=cols, x_row_stride=cols, scale_stride=cols)
    _refuse(lib, "dard_mx_quantize", _mx(), change, SHAPE)


@pytest.mark.parametrize("batch,rows,cols", [(0, 1 << 20, 32), (1 << 20, 0, 1 << 25)])
def test_quantize_of_nothing(lib, batch, rows, cols):  # noqa: F811
    a = _mx()
    a.batch, a.rows, a.cols, a.x_row_stride, a.scale_stride, a.x = batch, rows, cols, cols, cols, None
    assert lib.dard_mx_quantize(ctypes.byref(a), None) == 0
