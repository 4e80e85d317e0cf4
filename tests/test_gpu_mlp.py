"""The experts' MLP operators on the GPU against the float64 oracle.

Tolerances, derived from the arithmetic before any run:
* MXFP8 codes and scales of given values: equal (the rounding is exact).
* The norm in fp32: a thread adds up to 32 squares, then at most 10 pairwise steps, so the sum
  is off by at most 42 * 2^-24, its root by half that, and the reciprocal root (2 ulp), the
  scaling and the weight by 5 more roundings: 26 * 2^-24 < 2e-6 of a value; 4e-6 is asked. In
  bf16 half a unit in the last place of the result (8 bits: 2^(e - 9) for a value in
  [2^(e - 1), 2^e)) on top; as MXFP8 half a step of e4m3.
* Routing weights: an exponential of 2 ulp, at most 16 + 5 additions per sum, two divisions:
  30 * 2^-24 < 2e-6; 4e-6 is asked. Ids, offsets and rows: equal, with the deciding gaps of
  the inputs above 1e-6 (asserted on the oracle's side).
* The experts' products: the oracle's own elementwise bound (see there), and bf16's half unit.
"""
import numpy as np
import pytest
import torch

from oracle import mlp_oracle as O
from paper_2608_26574_gb300 import binding as B

pytestmark = pytest.mark.gpu

NORM_REL = 4e-6
ROUTE_REL = 4e-6
DEV = "cuda"


def _t(a, dtype="f32"):
    t = torch.from_numpy(np.ascontiguousarray(a, dtype=np.float32))
    return t.to(torch.bfloat16 if dtype == "bf16" else torch.float32).to(DEV)


def _np(t):
    return t.double().cpu().numpy()


def half_bf16(v):
    """Half a unit in the last place of bf16 at |v| (the next binade's where v rounds up to it)."""
    _, e = np.frexp(np.abs(v) * (1 + 2.0 ** -9))
    return np.ldexp(1.0, e - 9)


def _nan_equal(a, b):
    return np.array_equal(a, b, equal_nan=True)


# ---------------------------------------------------------------------------- MXFP8 rounding
def _values(rows, cols, seed, dtype):
    rng = np.random.default_rng(seed)
    v = rng.normal(size=(rows, cols)) * 2.0 ** rng.integers(-12, 12, (rows, 1))
    flat = v.reshape(-1)
    edge = [448.0, 1.75, -1.75, 1.7578125, 0.0, 2.0 ** -20, 464.0, -0.0]
    flat[::37] = np.resize(edge, flat[::37].shape)
    v = v.astype(np.float32)
    return O.round_bf16(v) if dtype == "bf16" else v.astype(np.float64)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("batch,rows,cols", [(1, 1, 32), (1, 5, 160), (3, 130, 96), (2, 128, 256),
                                             (1, 300, 1056)])
def test_quantize_both_layouts(dtype, batch, rows, cols):
    v = _values(batch * rows, cols, rows + cols, dtype).reshape(batch, rows, cols)
    x = _t(v, dtype)
    want, bytes_ = O.mx_round(v)
    for layout in (B.MX_SCALE_ROWS, B.MX_SCALE_TILES):
        codes = torch.full(x.shape, 3, dtype=torch.uint8, device=DEV)
        scales = torch.full(B.mx_scale_shape(x.shape, layout), 77, dtype=torch.uint8, device=DEV)
        B.dard_mx_quantize(x, codes, scales, layout)
        torch.cuda.synchronize()
        assert np.array_equal(_np(codes.view(torch.float8_e4m3fn)), want)
        s = scales.cpu().numpy()
        if layout == B.MX_SCALE_ROWS:
            assert np.array_equal(s[..., :cols // 32], bytes_)
            assert (s[..., cols // 32:] == 77).all()  # the pitch's rest is not written
        else:
            assert np.array_equal(s, np.stack([O.tile_scales(b) for b in bytes_]))


@pytest.mark.parametrize("offset,pad", [(0, 8), (1, 0), (3, 5)])
def test_quantize_strides_and_alignment(offset, pad):
    """Rows inside wider buffers, on and off 16-byte boundaries, and matrices apart."""
    v = _values(2 * 40, 64, offset + pad, "f32").reshape(2, 40, 64)
    buf = torch.full((2, 43, 64 + pad + offset), float("nan"), device=DEV)
    x = buf[:, 2:42, offset:offset + 64]
    x.copy_(_t(v))
    codes = torch.empty(2, 40, 64, dtype=torch.float8_e4m3fn, device=DEV)
    scales = torch.empty(B.mx_scale_shape(x.shape), dtype=torch.uint8, device=DEV)
    B.dard_mx_quantize(x, codes, scales)
    want, bytes_ = O.mx_round(v)
    assert np.array_equal(_np(codes), want)
    assert np.array_equal(scales.cpu().numpy()[..., :2], bytes_)


@pytest.mark.parametrize("vector", [True, False])
def test_quantize_infinities_and_nan(vector):
    v = np.ones((4, 96))
    v[0, 33], v[1, 0], v[2, 95], v[3, 64] = np.nan, np.inf, -np.inf, 3.0e38
    buf = torch.zeros(4, 96 + (0 if vector else 1), device=DEV)
    x = buf[:, -96:]
    x.copy_(_t(v))
    codes = torch.empty(4, 96, dtype=torch.float8_e4m3fn, device=DEV)
    scales = torch.empty(B.mx_scale_shape(x.shape), dtype=torch.uint8, device=DEV)
    B.dard_mx_quantize(x, codes, scales)
    want, bytes_ = O.mx_round(v.astype(np.float32))
    assert _nan_equal(_np(codes), want)
    assert np.array_equal(scales.cpu().numpy()[:, :3], bytes_)


def test_quantize_nothing():
    x = torch.empty(0, 64, device=DEV)
    B.dard_mx_quantize(x, torch.empty(0, 64, dtype=torch.uint8, device=DEV),
                       torch.empty(0, 16, dtype=torch.uint8, device=DEV))


# ---------------------------------------------------------------------------- residual + norm
def _norm_inputs(rows, dim, dtype, seed, delta=True, weight=True):
    rng = np.random.default_rng(seed)
    q = O.round_bf16 if dtype == "bf16" else lambda a: np.asarray(a, np.float32).astype(float)
    x = q(rng.normal(size=(rows, dim)) * 2.0 ** rng.integers(-6, 6, (1, dim)))
    d = q(rng.normal(size=(rows, dim))) if delta else None
    w = q(1 + 0.2 * rng.normal(size=dim)) if weight else None
    return x, d, w


def _check_norm(got, want, dtype):
    half = half_bf16(want) if dtype == "bf16" else 0.0
    assert _nan_equal(np.isnan(got), np.isnan(want))
    ok = np.abs(got - want) <= NORM_REL * np.abs(want) + half + 1e-37
    assert (ok | np.isnan(want)).all(), np.abs(got - want).max()


def _check_norm_mx(codes, scale_bytes, want):
    """Every value within half a step of e4m3 (plus the fp32 bound) of the exact one, under the
    scale that the exact block has, or, next to a boundary, its neighbour's."""
    _, bytes_ = O.mx_round(want)
    off = bytes_.astype(int) != scale_bytes
    top = np.abs(want).reshape(*want.shape[:-1], -1, 32).max(-1)
    edge = 448 * np.ldexp(1.0, np.minimum(bytes_, scale_bytes).astype(int) - 127)
    assert (np.abs(top - edge) <= NORM_REL * top)[off].all()
    s = np.repeat(np.ldexp(1.0, scale_bytes.astype(int) - 127), 32, -1)
    _, e = np.frexp(want / s)
    half = np.ldexp(1.0, np.maximum(e - 1, -6) - 4) * s
    assert (np.abs(codes * s - want) <= half * (1 + 1e-9) + NORM_REL * np.abs(want)).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,dim", [(1, 1), (3, 7), (1, 32), (5, 96), (6, 512), (2, 1000),
                                      (7, 1024), (3, 2048), (2, 4096), (3, 4100), (1, 8192),
                                      (2, 8200), (1, 16384), (1, 20000), (1, 32768)])
def test_norm_shapes(dtype, rows, dim):
    x, d, w = _norm_inputs(rows, dim, dtype, dim + rows)
    r, n = O.residual_norm(x, d, w, 1e-6, dtype == "bf16")
    X, D, W = _t(x, dtype), _t(d, dtype), _t(w, dtype)
    res, y = torch.empty_like(X), torch.empty_like(X)
    mx = dim % 32 == 0
    y8 = torch.empty(rows, dim, dtype=torch.float8_e4m3fn, device=DEV) if mx else None
    s8 = torch.empty(B.mx_scale_shape((rows, dim)), dtype=torch.uint8, device=DEV) if mx else None
    B.dard_residual_norm(X, D, W, 1e-6, residual=res, y=y, y8=y8, y8_scale=s8)
    torch.cuda.synchronize()
    assert np.array_equal(_np(res), r)
    _check_norm(_np(y), n, dtype)
    if mx:
        _check_norm_mx(_np(y8), s8.cpu().numpy()[:, :dim // 32], n)
    assert torch.equal(X, _t(x, dtype)) and torch.equal(D, _t(d, dtype))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("dim", [64, 1536])
@pytest.mark.parametrize("delta,weight,outs", [(False, False, "y"), (False, True, "8"),
                                               (True, False, "r"), (True, True, "ry"),
                                               (False, True, "r8")])
def test_norm_optional_parts(dtype, dim, delta, weight, outs):
    x, d, w = _norm_inputs(9, dim, dtype, 5, delta, weight)
    r, n = O.residual_norm(x, d, w, 1e-5, dtype == "bf16")
    X = _t(x, dtype)
    res = torch.empty_like(X) if "r" in outs else None
    y = torch.empty_like(X) if "y" in outs else None
    y8 = torch.empty(9, dim, dtype=torch.uint8, device=DEV) if "8" in outs else None
    s8 = torch.empty(B.mx_scale_shape((9, dim)), dtype=torch.float8_e8m0fnu, device=DEV) \
        if "8" in outs else None
    B.NormCall(dim, X.dtype, None if w is None else _t(w, dtype), 1e-5)(
        X, None if d is None else _t(d, dtype), res, y, y8, s8)
    if res is not None:
        assert np.array_equal(_np(res), r)
    if y is not None:
        _check_norm(_np(y), n, dtype)
    if y8 is not None:
        _check_norm_mx(_np(y8.view(torch.float8_e4m3fn)),
                       s8.view(torch.uint8).cpu().numpy()[:, :dim // 32], n)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("dim,offset,pad", [(256, 0, 8), (256, 1, 0), (96, 3, 7), (4096, 5, 0)])
def test_norm_strides_alignment_and_in_place(dtype, dim, offset, pad):
    """Rows inside wider buffers, on and off 16-byte boundaries; residual in place of x, y in
    place of delta; nothing outside the rows is touched."""
    x, d, w = _norm_inputs(11, dim, dtype, 8)
    r, n = O.residual_norm(x, d, w, 1e-6, dtype == "bf16")
    t = torch.bfloat16 if dtype == "bf16" else torch.float32

    def inside(v):
        buf = torch.full((11, offset + dim + pad), 5.0, dtype=t, device=DEV)
        buf[:, offset:offset + dim] = _t(v, dtype)
        return buf, buf[:, offset:offset + dim]

    xb, X = inside(x)
    db, D = inside(d)
    y8b = torch.full((11, dim + 32), 9, dtype=torch.uint8, device=DEV)
    s8 = torch.empty(B.mx_scale_shape((11, dim)), dtype=torch.uint8, device=DEV)
    B.dard_residual_norm(X, D, _t(w, dtype), residual=X, y=D, y8=y8b[:, :dim], y8_scale=s8)
    torch.cuda.synchronize()
    assert np.array_equal(_np(X), r)
    _check_norm(_np(D), n, dtype)
    _check_norm_mx(_np(y8b[:, :dim].contiguous().view(torch.float8_e4m3fn)),
                   s8.cpu().numpy()[:, :dim // 32], n)
    assert (y8b[:, dim:] == 9).all()
    for b in (xb, db):
        assert (b[:, :offset] == 5).all() and (b[:, offset + dim:] == 5).all()


@pytest.mark.parametrize("dim", [64, 99, 2048])
def test_norm_special_rows(dim):
    """Zero rows give zeros; a NaN or an infinity makes its row NaN and no other; rows whose
    squares leave fp32 give zeros (the sum is infinite) as in fp32 arithmetic."""
    x = np.ones((5, dim), np.float32)
    x[0] = 0
    x[1, dim // 2] = np.nan
    x[2, 0] = np.inf
    x[3] = 1e30
    X = _t(x)
    y = torch.empty_like(X)
    B.dard_residual_norm(X, y=y)
    got = _np(y)
    assert (got[0] == 0).all() and np.isnan(got[1]).all()
    # inf * (1 / inf) is NaN at the infinity, the others are divided to 0
    assert np.isnan(got[2, 0]) and (got[2, 1:] == 0).all()
    assert (got[3] == 0).all()
    assert np.allclose(got[4], 1 / np.sqrt(1 + 1e-6), rtol=1e-6)


def test_norm_nothing_and_another_stream():
    X = torch.empty(0, 64, device=DEV)
    B.dard_residual_norm(X, y=torch.empty_like(X))
    x, d, w = _norm_inputs(40, 512, "bf16", 3)
    s = torch.cuda.Stream()
    X, D, W = _t(x, "bf16"), _t(d, "bf16"), _t(w, "bf16")
    y = torch.empty_like(X)
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        B.dard_residual_norm(X, D, W, y=y)
    s.synchronize()
    _check_norm(_np(y), O.residual_norm(x, d, w, 1e-6, True)[1], "bf16")


# ---------------------------------------------------------------------------- routing
def _route(logits, dtype, top_k, plan=True, **kw):
    L = _t(logits, dtype)
    t, n = L.shape
    ids = torch.full((t, top_k), -7, dtype=torch.int32, device=DEV)
    w = torch.full((t, top_k), float("nan"), device=DEV)
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    offsets = torch.full((n + 1,), -7, dtype=torch.int32, device=DEV) if plan else None
    rows = torch.full((t * top_k,), -7, dtype=torch.int32, device=DEV) if plan else None
    ws = torch.full((max(B.dard_route_workspace_size(t, n, top_k), 16),), 255, dtype=torch.uint8,
                    device=DEV)
    bias = kw.pop("bias", None)
    B.dard_route(L, ids, w, top_k, bias=None if bias is None else _t(bias), offsets=offsets,
                 rows=rows, workspace=ws, status=status, **kw)
    torch.cuda.synchronize()
    return ids, w, offsets, rows, int(status.item())


def _check_route(logits, top_k, got, **kw):
    scoring = "sigmoid" if kw.pop("scoring", 0) == B.ROUTE_SIGMOID else "softmax"
    ids, w, invalid, gap = O.route(logits, top_k, scoring, **kw)
    assert gap > 1e-6  # the inputs decide every id beyond fp32's resolution
    gi, gw, go, gr, status = got
    assert np.array_equal(gi.cpu().numpy(), ids)
    assert (np.abs(_np(gw) - w) <= ROUTE_REL * np.abs(w)).all()
    if go is not None:
        offsets, rows = O.plan(ids, logits.shape[1])
        assert np.array_equal(go.cpu().numpy(), offsets)
        assert np.array_equal(gr.cpu().numpy(), rows)
    assert status == (B.STATUS_INVALID_ROW if invalid.any() else 0)


def _grid_logits(t, n, seed, levels=24):
    """Logits on a grid of quarters, off 0 by an eighth (so that no two sigmoids add up to 1):
    exact ties everywhere, and no near ones."""
    rng = np.random.default_rng(seed)
    return rng.integers(-levels, levels, (t, n)) / 4.0 + 0.125


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("scoring", [B.ROUTE_SOFTMAX, B.ROUTE_SIGMOID])
@pytest.mark.parametrize("t,n,k", [(1, 1, 1), (1, 64, 8), (3, 5, 5), (64, 33, 4), (65, 32, 1),
                                   (130, 160, 6), (400, 256, 8), (40, 512, 32), (170, 96, 11)])
def test_route_sizes_and_ties(dtype, scoring, t, n, k):
    logits = _grid_logits(t, n, t + n)
    for plan in (True, False):
        got = _route(logits, dtype, k, plan=plan, scoring=scoring, scale=1.5)
        _check_route(logits, k, got, scoring=scoring, scale=1.5)


@pytest.mark.parametrize("scoring", [B.ROUTE_SOFTMAX, B.ROUTE_SIGMOID])
@pytest.mark.parametrize("n,groups,top_groups,k", [(16, 4, 2, 3), (160, 8, 3, 6), (256, 8, 4, 8),
                                                   (24, 24, 5, 4), (96, 3, 1, 7), (512, 32, 9, 8),
                                                   (30, 5, 5, 6)])
def test_route_groups_and_bias(scoring, n, groups, top_groups, k):
    """Groups on coarse logits (exact ties of ranks and choices), then with a bias on random
    ones (a bias on coarse logits would give sums that are equal but for their rounding)."""
    rng = np.random.default_rng(n)
    kw = dict(scoring=scoring, groups=groups, top_groups=top_groups)
    logits = _grid_logits(150, n, n + groups, levels=3)
    _check_route(logits, k, _route(logits, "f32", k, **kw), **kw)
    logits = rng.normal(size=(150, n)).astype(np.float32)
    bias = (0.1 * rng.normal(size=n)).astype(np.float32)
    _check_route(logits, k, _route(logits, "f32", k, bias=bias, **kw), bias=bias, **kw)


@pytest.mark.parametrize("n", [31, 40, 90, 128, 150, 190, 200, 256, 270, 380, 400])
@pytest.mark.parametrize("k", [1, 2, 3, 9])
def test_route_expert_counts(n, k):
    """Every number of experts per lane, with ties."""
    for t in (31, 70):
        logits = _grid_logits(t, n, t + n + k)
        _check_route(logits, k, _route(logits, "f32", k))


@pytest.mark.parametrize("n", [20, 60, 100, 160, 256, 300, 512])
def test_route_choices_one_unit_apart(n):
    """Scores of exactly a half plus a bias of whole units in the last place of fp32: choices that
    differ in their last bits alone come out in their order, equal ones by expert."""
    k, t = min(n, 32), 40
    for spread in (n, n // 4):
        units = np.random.default_rng(n).integers(0, spread, n)
        ids, *_ = _route(np.zeros((t, n)), "f32", k, scoring=B.ROUTE_SIGMOID, bias=units * 2.0 ** -24)
        assert ids.tolist() == [np.argsort(-units, kind="stable")[:k].tolist()] * t


@pytest.mark.parametrize("t", [12, 200])
def test_route_masked_and_invalid_rows(t):
    """Experts switched off, tokens with fewer experts than slots, tokens with none, and tokens
    with NaN or +inf: no place of the plan is lost or doubled."""
    logits = _grid_logits(t, 48, t)
    rng = np.random.default_rng(t)
    logits[rng.random(logits.shape) < 0.5] = -np.inf
    logits[0] = -np.inf
    logits[1, 2:] = -np.inf
    logits[2, 47] = np.nan
    logits[3, 0] = np.inf
    logits[4, :] = -3.0e38
    for scoring in (B.ROUTE_SOFTMAX, B.ROUTE_SIGMOID):
        for kw in (dict(), dict(groups=6, top_groups=2)):
            got = _route(logits, "f32", 6, scoring=scoring, **kw)
            _check_route(logits, 6, got, scoring=scoring, **kw)


def test_route_without_renormalising_and_zero_sums():
    logits = _grid_logits(20, 16, 4)
    for scoring in (B.ROUTE_SOFTMAX, B.ROUTE_SIGMOID):
        got = _route(logits, "f32", 4, scoring=scoring, renormalise=False, scale=0.5)
        _check_route(logits, 4, got, scoring=scoring, renormalise=False, scale=0.5)
    low = np.full((2, 8), -500.0)  # sigmoids that are 0 in fp32: weights 0, not NaN
    ids, w, *_ = _route(low, "f32", 3, scoring=B.ROUTE_SIGMOID)
    assert ids.tolist() == [[0, 1, 2]] * 2 and (w == 0).all()


def test_route_row_stride_no_tokens_and_repeats():
    logits = _grid_logits(100, 40, 9)
    buf = torch.full((100, 47), float("nan"), device=DEV)
    buf[:, 3:43] = _t(logits)
    outs = []
    for L in (buf[:, 3:43], _t(logits), buf[:, 3:43]):
        ids = torch.empty(100, 4, dtype=torch.int32, device=DEV)
        w = torch.empty(100, 4, device=DEV)
        o = torch.empty(41, dtype=torch.int32, device=DEV)
        r = torch.empty(400, dtype=torch.int32, device=DEV)
        ws = torch.empty(B.dard_route_workspace_size(100, 40, 4), dtype=torch.uint8, device=DEV)
        B.dard_route(L, ids, w, 4, offsets=o, rows=r, workspace=ws)
        outs.append((ids, w, o, r))
    for other in outs[1:]:
        assert all(torch.equal(a, b) for a, b in zip(outs[0], other))
    o = torch.full((41,), 5, dtype=torch.int32, device=DEV)
    e = torch.empty(0, 4, dtype=torch.int32, device=DEV)
    B.dard_route(torch.empty(0, 40, device=DEV), e, torch.empty(0, 4, device=DEV), 4, offsets=o,
                 rows=torch.empty(0, dtype=torch.int32, device=DEV))
    assert (o == 0).all()


# ---------------------------------------------------------------------------- experts
def _experts_case(t, n, k, d, f, mx, seed, drop=0.1):
    rng = np.random.default_rng(seed)
    c = {}
    for name, shape in (("x", (t, d)), ("w1", (n, f, d)), ("w3", (n, f, d)), ("w2", (n, d, f))):
        v = rng.normal(size=shape) / (1.0 if name == "x" else np.sqrt(shape[-1]))
        if not mx:
            c[name] = O.round_bf16(v)
            continue
        codes, byte = O.mx_round(v * 2.0 ** rng.integers(-2, 3, (*shape[:-1], 1)))
        c[name], c[name + "_codes"], c[name + "_byte"] = O.mx_value(codes, byte), codes, byte
    ids = np.stack([rng.permutation(n)[:k] for _ in range(t)]).astype(np.int32).reshape(t, k)
    ids[rng.random((t, k)) < drop] = -1
    c["ids"], c["weights"] = ids, rng.random((t, k)).astype(np.float32)
    c["offsets"], c["rows"] = O.plan(ids, n)
    return c


def _run_experts(c, n, mx, y_dtype=torch.float32, x_pad=0, y_pad=0, status=None, ws=None):
    t, d = c["x"].shape
    k, f = c["ids"].shape[1], c["w1"].shape[1]
    dev = {m: torch.from_numpy(c[m]).to(DEV) for m in ("ids", "weights", "offsets", "rows")}
    if ws is None:  # scratch that holds NaN wherever it is read as anything
        ws = torch.full((max(B.dard_experts_workspace_size(t, n, k, d, f), 16),), 255,
                        dtype=torch.uint8, device=DEV)
    w = []
    for m in ("w1", "w3", "w2"):
        if mx:
            w.append(_t(c[m + "_codes"]).to(torch.float8_e4m3fn))
            w.append(torch.from_numpy(np.stack([O.tile_scales(b) for b in c[m + "_byte"]])).to(DEV))
        else:
            w += [_t(c[m], "bf16"), None]
    if mx:
        x = torch.full((t, d + x_pad), 0x7f, dtype=torch.uint8, device=DEV)  # NaN around the rows
        x[:, :d] = _t(c["x_codes"]).to(torch.float8_e4m3fn).view(torch.uint8)
        x = x[:, :d]
        xs = torch.full(B.mx_scale_shape((t, d)), 255, dtype=torch.uint8, device=DEV)
        xs[:, :d // 32] = torch.from_numpy(c["x_byte"]).to(DEV)
    else:
        x = torch.full((t, d + x_pad), float("nan"), dtype=torch.bfloat16, device=DEV)
        x[:, :d] = _t(c["x"], "bf16")
        x, xs = x[:, :d], None
    yb = torch.full((t, d + y_pad), float("nan"), dtype=y_dtype, device=DEV)
    B.dard_experts(x, xs, *w, dev["ids"], dev["weights"], dev["offsets"], dev["rows"], yb[:, :d],
                   ws, status)
    torch.cuda.synchronize()
    assert y_pad == 0 or torch.isnan(yb[:, d:]).all()
    return yb[:, :d]


def _check_experts(c, got, mx):
    y, tol = O.experts(c["x"], c["w1"], c["w3"], c["w2"], c["ids"], c["weights"], mx)
    if got.dtype == torch.bfloat16:
        tol = tol + half_bf16(np.abs(y) + tol)
    err = np.abs(_np(got) - y)
    assert (err <= tol + 1e-30).all(), (err.max(), (err / (tol + 1e-30)).max())


@pytest.mark.parametrize("mx", [True, False])
@pytest.mark.parametrize("t,n,k,d,f", [
    (1, 1, 1, 32, 32), (1, 8, 3, 64, 96), (3, 4, 4, 160, 32), (33, 8, 3, 96, 160),
    (128, 1, 1, 128, 128), (129, 1, 1, 256, 416), (200, 3, 2, 288, 224), (7, 40, 6, 544, 352),
    (300, 2, 1, 64, 1056), (2, 2, 2, 1056, 2080)])
def test_experts_shapes(mx, t, n, k, d, f):
    c = _experts_case(t, n, k, d, f, mx, t + d)
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    for y_dtype in (torch.float32, torch.bfloat16):
        _check_experts(c, _run_experts(c, n, mx, y_dtype, status=status), mx)
    assert int(status.item()) == 0


@pytest.mark.parametrize("mx", [True, False])
def test_experts_wide_tiles(mx):
    """Enough row tiles that both products take their wide tiles, with ragged last ones in rows
    and columns (checked on a sample of tokens: the oracle is slow)."""
    t, n, k, d, f = 2600, 40, 6, 608, 736
    c = _experts_case(t, n, k, d, f, mx, 77)
    got = _run_experts(c, n, mx)
    some = np.concatenate([np.arange(40), np.arange(t - 40, t)])
    part = dict(c, x=c["x"][some], ids=c["ids"][some], weights=c["weights"][some])
    _check_experts(part, got[torch.from_numpy(some).to(DEV)], mx)
    assert torch.isfinite(got).all()


@pytest.mark.parametrize("mx", [True, False])
def test_experts_skew_empty_and_strides(mx):
    """Every token to one expert of many, then no token to any, rows inside wider buffers."""
    c = _experts_case(150, 16, 2, 128, 192, mx, 5, drop=0.0)
    c["ids"][:] = [[9, 2]]
    c["offsets"], c["rows"] = O.plan(c["ids"], 16)
    _check_experts(c, _run_experts(c, 16, mx, x_pad=32, y_pad=8), mx)
    for k in (1, 2):
        e = _experts_case(20, 4, k, 64, 64, mx, 6, drop=1.1)
        assert (_run_experts(e, 4, mx, torch.bfloat16) == 0).all()


@pytest.mark.parametrize("mx", [True, False])
def test_experts_run_to_run_and_workspace_reuse(mx):
    """Equal bits from equal calls, whatever an earlier call left in the workspace."""
    a = _experts_case(190, 6, 3, 256, 320, mx, 11)
    b = _experts_case(61, 6, 2, 256, 320, mx, 12)
    ws = torch.full((B.dard_experts_workspace_size(190, 6, 3, 256, 320),), 255, dtype=torch.uint8,
                    device=DEV)
    first = _run_experts(a, 6, mx, ws=ws).clone()
    _check_experts(b, _run_experts(b, 6, mx, ws=ws), mx)
    assert torch.equal(_run_experts(a, 6, mx, ws=ws), first)


def test_experts_nan_reaches_its_own_token_only():
    """A NaN or an infinity in one token's input makes that token's outputs NaN, no other's."""
    c = _experts_case(40, 4, 2, 128, 128, True, 21, drop=0.0)
    want = _run_experts(c, 4, True)
    c["x_byte"] = c["x_byte"].copy()
    c["x_byte"][7, 1] = 255
    got = _run_experts(c, 4, True)
    assert torch.isnan(got[7]).all()
    keep = torch.arange(40, device=DEV) != 7
    assert torch.equal(got[keep], want[keep])


def test_experts_plan_that_is_none_stays_in_bounds():
    """Offsets that fall or pass the end and rows out of range: no access outside the buffers
    (clamped in the kernel), and the next call is right."""
    c = _experts_case(50, 4, 2, 64, 64, True, 31)
    bad = dict(c, offsets=np.array([0, 90, 10, 500, 100], np.int32),
               rows=np.where(np.arange(100) % 3 == 0, 1 << 30, c["rows"]).astype(np.int32))
    _run_experts(bad, 4, True)
    bad = dict(c, offsets=np.array([-5, 1 << 30, -9, 1 << 30, 7], np.int32))
    _run_experts(bad, 4, True)
    _check_experts(c, _run_experts(c, 4, True), True)


# ---------------------------------------------------------------------------- together
def test_norm_route_experts_in_a_graph():
    """The layer's order, captured once and replayed on new inputs: as the calls one by one."""
    t, n, k, d, f = 70, 16, 4, 256, 192
    g = torch.Generator(device=DEV).manual_seed(1)
    rn = lambda *s: torch.randn(*s, generator=g, device=DEV)  # noqa: E731
    w = []
    for shape in ((n, f, d), (n, f, d), (n, d, f)):
        codes = torch.empty(shape, dtype=torch.float8_e4m3fn, device=DEV)
        scales = torch.empty(B.mx_scale_shape(shape, B.MX_SCALE_TILES), dtype=torch.uint8, device=DEV)
        B.dard_mx_quantize(rn(*shape) / shape[-1] ** 0.5, codes, scales, B.MX_SCALE_TILES)
        w += [codes, scales]
    wr = rn(d, n).to(torch.bfloat16)
    x, delta = rn(t, d).to(torch.bfloat16), rn(t, d).to(torch.bfloat16)
    ws = torch.empty(B.dard_experts_workspace_size(t, n, k, d, f), dtype=torch.uint8, device=DEV)
    rws = torch.empty(max(B.dard_route_workspace_size(t, n, k), 16), dtype=torch.uint8, device=DEV)
    norm, route = B.NormCall(d, torch.bfloat16), B.RouteCall(n, k, workspace=rws)
    experts = B.ExpertsCall(*w, workspace=ws)
    buf = dict(res=torch.empty_like(x), y=torch.empty_like(x),
               y8=torch.empty(t, d, dtype=torch.float8_e4m3fn, device=DEV),
               s8=torch.empty(B.mx_scale_shape((t, d)), dtype=torch.uint8, device=DEV),
               logits=torch.empty(t, n, dtype=torch.bfloat16, device=DEV),
               ids=torch.empty(t, k, dtype=torch.int32, device=DEV),
               wt=torch.empty(t, k, device=DEV),
               off=torch.empty(n + 1, dtype=torch.int32, device=DEV),
               rows=torch.empty(t * k, dtype=torch.int32, device=DEV), out=torch.empty_like(x))

    def layer():
        norm(x, delta, buf["res"], buf["y"], buf["y8"], buf["s8"])
        torch.mm(buf["y"], wr, out=buf["logits"])
        route(buf["logits"], buf["ids"], buf["wt"], buf["off"], buf["rows"])
        experts(buf["y8"], buf["s8"], buf["ids"], buf["wt"], buf["off"], buf["rows"], buf["out"])

    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        layer()
    torch.cuda.current_stream().wait_stream(s)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        layer()
    for _ in range(2):
        x.copy_(rn(t, d))
        graph.replay()
        torch.cuda.synchronize()
        replayed = {m: b.clone() for m, b in buf.items()}
        layer()
        torch.cuda.synchronize()
        for m, b in buf.items():
            assert torch.equal(b.view(torch.uint8), replayed[m].view(torch.uint8)), m
        assert torch.isfinite(buf["out"]).all()
