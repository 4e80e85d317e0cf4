"""The experts' MLP operators on tensors of more than 2^31 elements: the rows at their ends (whose
offsets do not fit 32 bits) against calls on those rows alone, which the other tests check (rows
do not depend on one another, so both give the same bits), or against the oracle."""
import numpy as np
import pytest
import torch

from oracle import mlp_oracle as O
from paper_2608_26574_gb300 import binding as B

pytestmark = pytest.mark.gpu

DEV = "cuda"


@pytest.fixture(autouse=True)
def room():
    if torch.cuda.mem_get_info()[0] < 60 << 30:
        pytest.skip("needs 60 GB of free device memory")
    yield
    torch.cuda.empty_cache()


def _normal(*shape, seed=1, dtype=torch.bfloat16):
    g = torch.Generator(device=DEV).manual_seed(seed)
    return torch.empty(*shape, device=DEV, dtype=dtype).normal_(generator=g)


def _bits(t):
    return t.contiguous().view(torch.uint8)


@pytest.mark.parametrize("dim,pad", [(4096, 0), (4064, 1)])
def test_norm(dim, pad):
    rows, some = 2 ** 31 // dim + 77, 90
    x = _normal(rows, dim + pad)[:, :dim]
    y = torch.empty(rows, dim, device=DEV, dtype=torch.bfloat16)
    y8 = torch.empty(rows, dim, device=DEV, dtype=torch.float8_e4m3fn)
    s8 = torch.zeros(B.mx_scale_shape((rows, dim)), device=DEV, dtype=torch.uint8)
    B.dard_residual_norm(x, y=y, y8=y8, y8_scale=s8)
    for part in (slice(0, some), slice(rows - some, rows)):
        xp = x[part].clone()
        outs = [torch.empty_like(xp), torch.empty_like(y8[part]), torch.zeros_like(s8[part])]
        B.dard_residual_norm(xp, y=outs[0], y8=outs[1], y8_scale=outs[2])
        for a, b in zip((y, y8, s8), outs):
            # (a row's sum may be added up in another order where the layouts differ)
            if pad == 0:
                assert torch.equal(_bits(a[part]), _bits(b))
        assert torch.allclose(y[part].float(), outs[0].float(), rtol=2 ** -7, atol=0)


@pytest.mark.parametrize("layout", [B.MX_SCALE_ROWS, B.MX_SCALE_TILES])
def test_quantize(layout):
    batch, rows, cols = 131, 4096, 4096
    x = _normal(batch, rows, cols)
    codes = torch.empty(x.shape, device=DEV, dtype=torch.float8_e4m3fn)
    scales = torch.zeros(B.mx_scale_shape(x.shape, layout), device=DEV, dtype=torch.uint8)
    B.dard_mx_quantize(x, codes, scales, layout)
    for i in (0, batch - 1):
        c, s = torch.empty_like(codes[i:i + 1]), torch.zeros_like(scales[i:i + 1])
        B.dard_mx_quantize(x[i:i + 1].clone(), c, s, layout)
        assert torch.equal(_bits(codes[i:i + 1]), _bits(c)) and torch.equal(scales[i:i + 1], s)


def test_route():
    n, k, some = 512, 3, 300
    t = 2 ** 31 // n + 1000
    logits = _normal(t, n)

    def route(x):
        out = [torch.empty(len(x), k, dtype=torch.int32, device=DEV), torch.empty(len(x), k, device=DEV),
               torch.empty(n + 1, dtype=torch.int32, device=DEV),
               torch.empty(len(x) * k, dtype=torch.int32, device=DEV)]
        ws = torch.empty(max(B.dard_route_workspace_size(len(x), n, k), 16), dtype=torch.uint8,
                         device=DEV)
        B.dard_route(x, out[0], out[1], k, offsets=out[2], rows=out[3], workspace=ws)
        return out

    ids, weights, offsets, rows = route(logits)
    for part in (slice(0, some), slice(t - some, t)):
        want = route(logits[part].clone())
        assert torch.equal(ids[part], want[0]) and torch.equal(weights[part], want[1])
    # the plan: a stable sort of the pairs by expert
    assert torch.equal(offsets[1:].long(), torch.bincount(ids.reshape(-1).long(), minlength=n).cumsum(0))
    assert torch.equal(rows.long(), torch.sort(ids.reshape(-1), stable=True).indices)


def _plan(ids, n):
    flat = ids.reshape(-1)
    counts = torch.bincount(flat.long(), minlength=n).cumsum(0)
    offsets = torch.cat([counts.new_zeros(1), counts]).to(torch.int32)
    return offsets, torch.sort(flat, stable=True).indices.to(torch.int32)


def _experts(x, w, ids, weights, n):
    t, d, f = *x.shape, w[0].shape[1]
    offsets, rows = _plan(ids, n)
    ws = torch.empty(B.dard_experts_workspace_size(t, n, ids.shape[1], d, f), dtype=torch.uint8,
                     device=DEV)
    y = torch.empty(t, d, device=DEV)
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    B.dard_experts(x, None, w[0], None, w[1], None, w[2], None, ids, weights, offsets, rows, y, ws,
                   status)
    torch.cuda.synchronize()
    assert int(status.item()) == 0
    return y


@pytest.mark.parametrize("t", [20, 300])
def test_experts_weights(t):
    """The last two of 130 experts of 4096 x 4096, in every matrix behind 2^31 elements."""
    n, d, f = 130, 4096, 4096
    w = [torch.zeros(n, *s, device=DEV, dtype=torch.bfloat16) for s in ((f, d), (f, d), (d, f))]
    for i, m in enumerate(w):
        m[128:] = _normal(2, *m.shape[1:], seed=i) / 64
    x = _normal(t, d, seed=9)
    ids = 128 + torch.arange(t, device=DEV, dtype=torch.int32)[:, None] % 2
    weights = torch.rand(t, 1, device=DEV)
    got = _experts(x, w, ids, weights, n)
    some = torch.arange(10, device=DEV) * (t - 1) // 9  # (the oracle is slow)
    np64 = [m.double().cpu().numpy() for m in (x[some], w[0][128:], w[1][128:], w[2][128:])]
    y, tol = O.experts(*np64, (ids[some] - 128).cpu().numpy(), weights[some].cpu().numpy(), False)
    assert (np.abs(got[some].double().cpu().numpy() - y) <= tol).all() and np.abs(y).mean() > 0.01


def test_experts_products():
    """More than 2^31 products of pairs before their sum: 128 times the same 64 tokens."""
    n, k, d, f, block = 8, 8, 32832, 64, 64
    w = [_normal(n, f, d, seed=1) / 181, _normal(n, f, d, seed=2) / 181, _normal(n, d, f, seed=3) / 8]
    x = _normal(block, d, seed=4).repeat(128, 1)
    ids = torch.stack([torch.randperm(n, device=DEV) for _ in range(block)]).to(torch.int32)
    weights = torch.rand(block, k, device=DEV)
    y = _experts(x, w, ids.repeat(128, 1), weights.repeat(128, 1), n)
    assert y.abs().mean() > 0.01
    assert torch.equal(y.view(128, block, d), y[:block].expand(128, block, d))
