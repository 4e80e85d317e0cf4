"""Each variant of dard_experts' kernels (few tokens; single CTAs; CTA pairs; pairs in one product and
single CTAs in the other), at the places where it can go wrong: ragged tiles, slots without an
expert, products written straight to y or through a split reduction, rows inside wider buffers,
NaN, plans that are none, and equal bits from equal calls. Values are held against the float64 oracle
under its own elementwise bound (and bf16's half unit), as in the other tests of the products."""
import numpy as np
import pytest
import torch

from paper_2608_26574_gb300 import binding as B

from .test_gpu_mlp import _check_experts, _experts_case, _run_experts

pytestmark = pytest.mark.gpu

DEV = "cuda"
# (tokens, experts, slots, dim, hidden): the sizes that make_plan in dard_experts.cu answers on
# 152 SMs with few; single; pairs
FEW, SINGLE, PAIRS = (20, 4, 2, 64, 96), (50, 4, 2, 64, 96), (200, 40, 2, 512, 256)


def _check_some(c, got, mx, count=14):
    """The oracle on some tokens, the first and the last among them (it is slow)."""
    t = len(c["x"])
    some = np.unique(np.r_[np.arange(count // 2), np.linspace(0, t - 1, count).astype(int)])
    part = dict(c, **{m: c[m][some] for m in ("x", "ids", "weights")})
    _check_experts(part, got[torch.from_numpy(some).to(DEV)], mx)


@pytest.mark.parametrize("mx", [True, False])
@pytest.mark.parametrize("y_dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("t,n,k,d,f", [
    (800, 1, 1, 4096, 1312),   # pairs, y written by the product, x copied by several warps per row
    (790, 1, 1, 4128, 1376),   # the same with ragged columns
    (700, 1, 1, 4128, 1280),   # single CTAs, then pairs
    (300, 2, 1, 96, 1760),     # pairs, then single CTAs with a reduction in three runs
    (170, 2, 2, 96, 1760),     # the same, two slots
    (300, 2, 1, 3360, 96),     # single CTAs, then pairs; y written by the product
    (170, 2, 2, 3360, 96),     # the same, two slots
    (200, 40, 2, 544, 288),    # pairs of tiles of which most have no rows
])
def test_variants_and_their_mixes(mx, y_dtype, t, n, k, d, f):
    c = _experts_case(t, n, k, d, f, mx, t + f, drop=0.1)
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    got = _run_experts(c, n, mx, y_dtype, x_pad=32, y_pad=16, status=status)
    assert int(status.item()) == 0
    _check_some(c, got, mx)
    assert torch.isfinite(got).all()
    none = torch.from_numpy((c["ids"] < 0).all(1)).to(DEV)
    assert (got[none] == 0).all()


@pytest.mark.parametrize("mx", [True, False])
@pytest.mark.parametrize("shape", [FEW, SINGLE, PAIRS, (300, 2, 2, 96, 1760), (300, 2, 2, 3360, 96)])
def test_equal_bits_whatever_the_workspace_held(mx, shape):
    t, n, k, d, f = shape
    c = _experts_case(t, n, k, d, f, mx, 61)
    size = B.dard_experts_workspace_size(t, n, k, d, f)
    first = None
    for fill in (255, 0, 127, 255):
        ws = torch.full((size,), fill, dtype=torch.uint8, device=DEV)
        for _ in range(4):
            got = _run_experts(c, n, mx, ws=ws)
            first = got if first is None else first
            assert torch.equal(got, first)


@pytest.mark.parametrize("shape", [FEW, SINGLE, PAIRS])
def test_nan_reaches_its_own_token_only(shape):
    t, n, k, d, f = shape
    c = _experts_case(t, n, k, d, f, True, 62, drop=0.0)
    want = _run_experts(c, n, True)
    c["x_byte"] = c["x_byte"].copy()
    c["x_byte"][7, 1] = 255
    got = _run_experts(c, n, True)
    assert torch.isnan(got[7]).all()
    keep = torch.arange(t, device=DEV) != 7
    assert torch.equal(got[keep], want[keep])


@pytest.mark.parametrize("mx", [True, False])
@pytest.mark.parametrize("shape", [FEW, SINGLE, PAIRS])
def test_plans_that_are_none_stay_in_bounds(mx, shape):
    """Offsets that fall or pass the end and rows out of range (clamped and skipped in the kernels),
    with nothing written around y; the next call is right."""
    t, n, k, d, f = shape
    c = _experts_case(t, n, k, d, f, mx, 63)
    pairs = t * k
    rng = np.random.default_rng(2)
    plans = [dict(offsets=np.resize([0, pairs - 10, 10, 5 * pairs], n + 1).astype(np.int32),
                  rows=np.where(np.arange(pairs) % 3 == 0, 1 << 30, c["rows"]).astype(np.int32)),
             dict(offsets=np.resize([-5, 1 << 30, -9], n + 1).astype(np.int32)),
             dict(offsets=np.full(n + 1, pairs, np.int32)),
             dict(rows=rng.integers(-9, 2 * pairs, pairs).astype(np.int32))]
    for bad in plans:
        _run_experts(dict(c, **bad), n, mx, y_pad=8)
    _check_some(c, _run_experts(c, n, mx), mx)
