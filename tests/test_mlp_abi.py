"""Refusals of the experts' MLP entry points: every argument that the library or the binding
turns down, on the host, before any launch (no GPU needed: the pointers are never followed)."""
import ctypes

import pytest
import torch

from paper_2608_26574_gb300 import binding as B
from paper_2608_26574_gb300 import build as BUILD

NULL, SHAPE, VALUE, CUDA, ALIGN, WORKSPACE = 1, 2, 3, 5, 6, 7
PTR = 0x10000


@pytest.fixture(scope="module")
def lib():
    BUILD.build()
    return B.lib()


def _refuse(lib, fn, args, change, code):
    for k, v in change.items():
        setattr(args, k, v)
    assert getattr(lib, fn)(ctypes.byref(args), None) == code
    assert lib.dard_last_error().decode() != ""


@pytest.mark.parametrize("fn", ["dard_residual_norm", "dard_mx_quantize", "dard_route",
                                "dard_experts"])
def test_null_args(lib, fn):
    assert getattr(lib, fn)(None, None) == NULL


def _norm():
    a = B.NormArgs()
    a.x, a.y, a.y8, a.y8_scale, a.residual = PTR, 2 * PTR, 3 * PTR, 4 * PTR, 5 * PTR
    a.dtype, a.dim, a.rows, a.eps = B.DARD_BF16, 64, 4, 1e-6
    a.x_stride = a.y_stride = a.y8_stride = a.residual_stride = 64
    a.y8_scale_stride = 16
    return a


@pytest.mark.parametrize("change,code", [
    ({"x": None}, NULL), ({"y": None, "y8": None, "residual": None}, NULL),
    ({"y8_scale": None}, NULL), ({"rows": -1}, SHAPE), ({"rows": 1 << 31}, SHAPE),
    ({"dim": 0}, SHAPE), ({"dim": B.NORM_MAX_DIM + 32}, SHAPE),
    ({"dim": 40}, SHAPE), ({"x_stride": 63}, SHAPE), ({"y_stride": 0}, SHAPE),
    ({"delta": PTR, "delta_stride": 8}, SHAPE), ({"residual_stride": 1}, SHAPE),
    ({"y8_stride": 32}, SHAPE), ({"y8_scale_stride": 1}, SHAPE), ({"dtype": 2}, VALUE),
    ({"eps": -1.0}, VALUE), ({"eps": float("nan")}, VALUE), ({"eps": float("inf")}, VALUE),
    ({"residual": 2 * PTR}, VALUE), ({"x": PTR + 1}, ALIGN), ({"weight": PTR + 1}, ALIGN),
    ({"y8_scale_stride": 8}, ALIGN), ({"y8_scale": PTR + 8}, ALIGN)])
def test_norm_refusals(lib, change, code):
    _refuse(lib, "dard_residual_norm", _norm(), change, code)


def _mx():
    a = B.MxArgs()
    a.x, a.codes, a.scales, a.dtype, a.layout = PTR, 2 * PTR, 3 * PTR, B.DARD_F32, B.MX_SCALE_ROWS
    a.batch, a.rows, a.cols, a.x_row_stride, a.x_batch_stride, a.scale_stride = 1, 4, 64, 64, 0, 16
    return a


@pytest.mark.parametrize("change,code", [
    ({"x": None}, NULL), ({"codes": None}, NULL), ({"scales": None}, NULL), ({"batch": -1}, SHAPE),
    ({"rows": -1}, SHAPE), ({"cols": 0}, SHAPE), ({"cols": 48}, SHAPE), ({"rows": 1 << 41}, SHAPE),
    ({"rows": 1 << 40}, SHAPE), ({"x_row_stride": 63}, SHAPE), ({"x_batch_stride": -1}, SHAPE),
    ({"scale_stride": 1}, SHAPE), ({"dtype": 2}, VALUE), ({"layout": 2}, VALUE),
    ({"x": PTR + 2}, ALIGN), ({"codes": PTR + 8}, ALIGN), ({"scales": PTR + 4}, ALIGN),
    ({"scale_stride": 8}, ALIGN)])
def test_quantize_refusals(lib, change, code):
    _refuse(lib, "dard_mx_quantize", _mx(), change, code)


def _route():
    a = B.RouteArgs()
    a.logits, a.ids, a.weights, a.offsets, a.rows = (PTR,) * 5
    a.logits_stride, a.dtype, a.scoring = 16, B.DARD_F32, B.ROUTE_SOFTMAX
    a.tokens, a.experts, a.top_k, a.groups, a.top_groups = 4, 16, 2, 1, 1
    a.renormalise, a.scale = 1, 1.0
    return a


@pytest.mark.parametrize("change,code", [
    ({"logits": None}, NULL), ({"ids": None}, NULL), ({"weights": None}, NULL),
    ({"offsets": None}, NULL), ({"rows": None}, NULL), ({"tokens": -1}, SHAPE),
    ({"experts": 0}, SHAPE), ({"experts": 513}, SHAPE), ({"top_k": 0}, SHAPE),
    ({"top_k": 17}, SHAPE), ({"experts": 64, "logits_stride": 64, "top_k": 33}, SHAPE),
    ({"tokens": (1 << 31) - 1}, SHAPE), ({"groups": 0}, SHAPE), ({"groups": 3}, SHAPE),
    ({"experts": 64, "logits_stride": 64, "groups": 64}, SHAPE), ({"top_groups": 0}, SHAPE),
    ({"groups": 4, "top_groups": 5}, SHAPE), ({"logits_stride": 15}, SHAPE), ({"dtype": 2}, VALUE),
    ({"scoring": 2}, VALUE), ({"renormalise": 2}, VALUE), ({"scale": float("nan")}, VALUE),
    ({"logits": PTR + 2}, ALIGN), ({"tokens": 100000}, WORKSPACE),
    ({"tokens": 100000, "workspace": PTR, "workspace_bytes": 8}, WORKSPACE),
    ({"tokens": 100000, "workspace": PTR + 1, "workspace_bytes": 1 << 30}, ALIGN)])
def test_route_refusals(lib, change, code):
    _refuse(lib, "dard_route", _route(), change, code)


def _experts():
    a = B.ExpertsArgs()
    for n in ("x", "x_scale", "w1", "w3", "w2", "w1_scale", "w3_scale", "w2_scale", "ids", "weights",
              "offsets", "rows", "y", "workspace"):
        setattr(a, n, PTR)
    a.dtype, a.y_dtype = B.DARD_MXFP8, B.DARD_BF16
    a.tokens, a.experts, a.top_k, a.dim, a.hidden = 4, 8, 2, 64, 96
    a.x_stride = a.y_stride = 64
    a.x_scale_stride = 16
    a.workspace_bytes = 1 << 30
    return a


@pytest.mark.parametrize("change,code", [
    *[({n: None}, NULL) for n in ("x", "x_scale", "w1", "w3", "w2", "w1_scale", "w3_scale",
                                  "w2_scale", "ids", "weights", "offsets", "rows", "y")],
    ({"workspace": None}, WORKSPACE), ({"workspace_bytes": 64}, WORKSPACE),
    ({"tokens": -1}, SHAPE), ({"tokens": 1 << 24}, SHAPE), ({"experts": 0}, SHAPE),
    ({"experts": 513}, SHAPE), ({"top_k": 0}, SHAPE), ({"top_k": 9}, SHAPE), ({"dim": 48}, SHAPE),
    ({"dim": 0}, SHAPE), ({"hidden": 16}, SHAPE), ({"hidden": 65568}, SHAPE), ({"x_stride": 32}, SHAPE),
    ({"y_stride": 32}, SHAPE), ({"x_scale_stride": 1}, SHAPE), ({"dtype": 0}, VALUE),
    ({"dtype": 3}, VALUE), ({"y_dtype": 2}, VALUE),
    *[({n: PTR + 8}, ALIGN) for n in ("x", "x_scale", "w1", "w3", "w2", "w1_scale", "w3_scale",
                                      "w2_scale", "y", "workspace")],
    ({"x_stride": 72}, ALIGN), ({"y_stride": 66}, ALIGN), ({"x_scale_stride": 8}, ALIGN)])
def test_experts_refusals(lib, change, code):
    _refuse(lib, "dard_experts", _experts(), change, code)


def test_nothing_to_do_is_no_error(lib):
    """No rows: success without a launch (there is no device here), whatever the pointers."""
    a = _norm()
    a.rows, a.x = 0, None
    assert lib.dard_residual_norm(ctypes.byref(a), None) == 0
    a = _mx()
    a.rows, a.x = 0, None
    assert lib.dard_mx_quantize(ctypes.byref(a), None) == 0
    a = _experts()
    a.tokens, a.x, a.workspace = 0, None, None
    assert lib.dard_experts(ctypes.byref(a), None) == 0
    a = _route()
    a.tokens, a.offsets, a.rows = 0, None, None
    assert lib.dard_route(ctypes.byref(a), None) == 0


def test_workspace_sizes(lib):
    assert B.dard_route_workspace_size(1, 64, 8) == 0
    assert B.dard_route_workspace_size(5000, 64, 8) > 0
    assert B.dard_route_workspace_size(5000, 64, 65) == 0
    assert B.dard_experts_workspace_size(0, 8, 2, 64, 96) == 0
    assert B.dard_experts_workspace_size(4, 8, 2, 65, 96) == 0
    # the product in between in bf16 and the pairs' products
    assert B.dard_experts_workspace_size(1000, 8, 2, 64, 96) >= 2000 * 96 * 2 + 2000 * 64 * 2


def test_scale_shapes():
    assert B.mx_scale_shape((5, 64)) == (5, 16)
    assert B.mx_scale_shape((2, 5, 1056)) == (2, 5, 48)
    assert B.mx_scale_shape((3, 129, 160), B.MX_SCALE_TILES) == (3, 2, 2, 512)
    with pytest.raises(ValueError):
        B.mx_scale_shape((5, 40))


def test_binding_refuses_before_the_library(lib):
    """Host tensors, wrong types and wrong shapes raise ValueError in the binding."""
    x = torch.zeros(4, 64)
    with pytest.raises(ValueError, match="device tensor"):
        B.dard_residual_norm(x, y=torch.zeros_like(x))
    with pytest.raises(ValueError, match="unsupported dtype"):
        B.NormCall(64, torch.float16)
    with pytest.raises(ValueError, match="device tensor"):
        B.dard_mx_quantize(x, x, x)
    with pytest.raises(ValueError, match="expected"):
        B.RouteCall(64, 2)(torch.zeros(4, 32), None, None)
    w = torch.zeros(2, 96, 64, dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="w1 and w3"):
        B.ExpertsCall(w, None, w, None, w, None, None)
