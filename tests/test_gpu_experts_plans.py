"""dard_experts on plans other than a router's ordinary ones, in every variant of its kernels, against
the float64 oracle under its own elementwise bound: tokens that name an expert in several slots, and calls where no token has an expert."""
import numpy as np
import pytest
import torch

from oracle import mlp_oracle as O
from paper_2608_26574_gb300 import binding as B

from .test_gpu_mlp import _check_experts, _experts_case, _run_experts

pytestmark = pytest.mark.gpu

DEV = "cuda"


@pytest.mark.parametrize("mx", [True, False])
@pytest.mark.parametrize("t,n,k,d,f", [(32, 4, 4, 160, 96), (32, 40, 9, 96, 288), (17, 3, 2, 288, 544),
                                       (33, 4, 4, 160, 96), (120, 5, 3, 64, 160)])
def test_a_token_names_an_expert_in_several_slots(mx, t, n, k, d, f):
    """Experts with more rows than there are tokens: all slots of all tokens to one expert, then
    two experts, then some slots without any."""
    c = _experts_case(t, n, k, d, f, mx, 3 * t + n, drop=0.0)
    rng = np.random.default_rng(t)
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    for ids in (np.full((t, k), n - 1), rng.integers(0, 2, (t, k)),
                np.where(rng.random((t, k)) < 0.1, -1, rng.integers(1, 3, (t, k)))):
        c["ids"] = ids.astype(np.int32)
        c["offsets"], c["rows"] = O.plan(c["ids"], n)
        _check_experts(c, _run_experts(c, n, mx, status=status), mx)
    assert int(status.item()) == 0


@pytest.mark.parametrize("mx", [True, False])
@pytest.mark.parametrize("t,n,k", [(400, 40, 1), (200, 40, 2)])
def test_no_token_has_an_expert_in_calls_of_cta_pairs(mx, t, n, k):
    """Sizes whose products run in pairs of CTAs, with x copied into the plan's order by a launch
    of its own: zeros, call after call, each with another plan in the same tensors right behind
    it on the stream, whose outputs are those of the same call alone."""
    d, f = 512, 256
    full = _experts_case(t, n, k, d, f, mx, 41, drop=0.0)
    want = _run_experts(full, n, mx, torch.float32)
    w = []
    for m in ("w1", "w3", "w2"):
        v = torch.from_numpy(full[m]).to(DEV)
        if not mx:
            w += [v.to(torch.bfloat16), None]
            continue
        codes = torch.from_numpy(full[m + "_codes"]).to(DEV).float().to(torch.float8_e4m3fn)
        tiles = np.stack([O.tile_scales(b) for b in full[m + "_byte"]])
        w += [codes, torch.from_numpy(tiles).to(DEV)]
    ws = torch.empty(B.dard_experts_workspace_size(t, n, k, d, f), dtype=torch.uint8, device=DEV)
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    call = B.ExpertsCall(*w, workspace=ws, status=status)
    if mx:
        x = torch.from_numpy(full["x_codes"]).to(DEV).float().to(torch.float8_e4m3fn)
        xs = torch.zeros(B.mx_scale_shape((t, d)), dtype=torch.uint8, device=DEV)
        xs[:, :d // 32] = torch.from_numpy(full["x_byte"]).to(DEV)
    else:
        x, xs = torch.from_numpy(full["x"]).to(DEV).to(torch.bfloat16), None
    plans = {}
    for name in ("none", "full"):
        ids = full["ids"] if name == "full" else np.full((t, k), -1, np.int32)
        plans[name] = [torch.from_numpy(a).to(DEV) for a in (ids, *O.plan(ids, n))]
    ids, offsets, rows = (torch.empty_like(a) for a in plans["none"])
    weights = torch.from_numpy(full["weights"]).to(DEV)
    ys = [torch.full((t, d), float("nan"), device=DEV) for _ in range(40)]
    for i, y in enumerate(ys):
        for to, a in zip((ids, offsets, rows), plans["full" if i % 2 else "none"]):
            to.copy_(a)
        call(x, xs, ids, weights, offsets, rows, y)
    torch.cuda.synchronize()
    assert int(status.item()) == 0
    for i, y in enumerate(ys):
        assert torch.equal(y, want if i % 2 else torch.zeros_like(y))
