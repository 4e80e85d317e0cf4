"""The experts' MLP entry points at and past the ends of their sizes, on the host (no GPU needed: the
pointers are never followed)."""
import ctypes

import pytest
import torch

from paper_2608_26574_gb300 import binding as B
from paper_2608_26574_gb300.experts import ExpertMLP

from .test_mlp_abi import (ALIGN, SHAPE, WORKSPACE, _experts, _mx, _refuse, _route,
                           lib)  # noqa: F401 (lib: a fixture)


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


@pytest.mark.parametrize("experts,top_k", [(1, 1), (64, 8), (256, 8), (512, 32)])
def test_route_workspace_serves_every_smaller_count(lib, experts, top_k):  # noqa: F811
    """A workspace for a token count is large enough for each count below it: the size never falls
    as the count rises, and a call accepts it (it is refused with a byte less than it needs, and
    with this much gets as far as the next check)."""
    counts = [*range(0, 6000), *range(6000, 40000, 37), (1 << 31) // top_k - 1]
    sizes = [B.dard_route_workspace_size(t, experts, top_k) for t in counts]
    assert all(a <= b for a, b in zip(sizes, sizes[1:]))
    assert sizes[0] == sizes[32] == 0 and sizes[33] > 0
    for t, size in list(zip(counts, sizes))[33::101]:
        a = _route()
        a.experts, a.top_k, a.tokens, a.logits_stride = experts, top_k, t, experts
        _refuse(lib, "dard_route", a, dict(workspace_bytes=size, workspace=8), ALIGN)
        _refuse(lib, "dard_route", a, dict(workspace_bytes=15), WORKSPACE)


@pytest.mark.parametrize("experts,top_k,dim,hidden", [
    (1, 1, 4096, 12288), (1, 1, 32, 65536), (64, 8, 2048, 1024), (8, 2, 96, 32768), (40, 6, 2208, 736),
    (512, 32, 256, 64), (6, 2, 64, 96), (3, 3, 128, 8192)])
def test_experts_workspace_serves_every_smaller_count(lib, experts, top_k, dim, hidden):  # noqa: F811
    """As for routing: the size never falls as the count rises, and calls accept it."""
    counts = [*range(0, 2600), *range(2600, 20000, 91), (1 << 24) // top_k]
    sizes = [B.dard_experts_workspace_size(t, experts, top_k, dim, hidden) for t in counts]
    assert sizes[0] == 0 and all(a <= b for a, b in zip(sizes, sizes[1:]))
    for dtype in (B.DARD_MXFP8, B.DARD_BF16):
        for t, size in list(zip(counts, sizes))[1::37]:
            a = _experts()
            a.dtype, a.tokens, a.experts, a.top_k, a.dim, a.hidden = dtype, t, experts, top_k, dim, hidden
            a.x_stride, a.y_stride, a.x_scale_stride = dim, dim, (dim + 511) // 512 * 16
            _refuse(lib, "dard_experts", a, dict(workspace_bytes=size, workspace=8), ALIGN)


@pytest.mark.parametrize("mx", [True, False])
def test_a_layer_of_host_tensors_is_refused(mx):
    w = torch.zeros(2, 96, 64, dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="device tensor"):
        ExpertMLP(w, w, w.mT.contiguous(), torch.zeros(64, 2, dtype=torch.bfloat16), 1, mx=mx)
