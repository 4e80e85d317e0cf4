"""The experts' MLP operators at the ends of the sizes that include/dard.h accepts."""
import math

import numpy as np
import pytest
import torch

from oracle import mlp_oracle as O
from paper_2608_26574_gb300 import binding as B

pytestmark = pytest.mark.gpu

DEV = "cuda"


def test_route_the_most_tokens():
    """2^31 - 1 tokens of one expert, two of them with the expert switched off: ids, weights and
    the plan, whose last places are the last that 32 bits hold."""
    if torch.cuda.mem_get_info()[0] < 60 << 30:
        pytest.skip("needs 60 GB of free device memory")
    t = 2 ** 31 - 1
    off = (5, t - 3)
    logits = torch.zeros(t, 1, dtype=torch.bfloat16, device=DEV)
    for i in off:
        logits[i] = -math.inf
    ids = torch.full((t, 1), 9, dtype=torch.int32, device=DEV)
    weights = torch.full((t, 1), 9.0, device=DEV)
    offsets = torch.full((2,), 9, dtype=torch.int32, device=DEV)
    rows = torch.full((t,), 9, dtype=torch.int32, device=DEV)
    ws = torch.empty(B.dard_route_workspace_size(t, 1, 1), dtype=torch.uint8, device=DEV)
    B.dard_route(logits, ids, weights, 1, offsets=offsets, rows=rows, workspace=ws)
    assert offsets.tolist() == [0, t - 2]
    assert rows[-2:].tolist() == [-1, -1]
    for i in off:
        assert ids[i].item() == -1 and weights[i].item() == 0
        ids[i], weights[i] = 0, 1
    step = 1 << 27
    for a in range(0, t, step):
        assert (ids[a:a + step] == 0).all() and (weights[a:a + step] == 1).all()
        want = torch.arange(a, min(a + step, t - 2), device=DEV)
        for i in off:
            want += want >= i
        assert torch.equal(rows[a:a + len(want)], want.to(torch.int32))


def test_route_one_workspace_for_every_count_below():
    """One RouteCall with the workspace of its most tokens, over counts on both sides of where a
    CTA begins to take more than 32 of them."""
    n, k, sms = 64, 4, torch.cuda.get_device_properties(0).multi_processor_count
    most = 32 * sms + 1
    ws = torch.empty(B.dard_route_workspace_size(most, n, k), dtype=torch.uint8, device=DEV)
    call = B.RouteCall(n, k, workspace=ws)
    g = torch.Generator(device=DEV).manual_seed(3)
    logits = torch.rand(most, n, generator=g, device=DEV).argsort(1) / 8.0  # no two alike in a row
    for t in (most, most - 1, most - 32, 33, 32, 1, 0):
        ids = torch.empty(t, k, dtype=torch.int32, device=DEV)
        weights = torch.empty(t, k, device=DEV)
        offsets = torch.empty(n + 1, dtype=torch.int32, device=DEV)
        rows = torch.empty(t * k, dtype=torch.int32, device=DEV)
        call(logits[:t], ids, weights, offsets, rows)
        assert torch.equal(ids, torch.topk(logits[:t], k).indices.to(torch.int32))
        want = O.plan(ids.cpu().numpy(), n)
        assert np.array_equal(offsets.cpu().numpy(), want[0])
        assert np.array_equal(rows.cpu().numpy(), want[1])
