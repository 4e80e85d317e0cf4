"""dard_experts on plans other than a router's ordinary ones, in every variant of its kernels, against
the float64 oracle under its own elementwise bound: tokens that name an expert in several slots."""
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
