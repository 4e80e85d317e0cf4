"""The experts' MLP operators at the ends of the sizes that include/dard.h accepts."""
import math

import pytest
import torch

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
