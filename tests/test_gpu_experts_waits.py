"""Waits of dard_experts' CTA pairs that run out at other places than a call's first stages: both
CTAs' copies report to one CTA's barriers, and those in flight are waited for before either CTA
ends. As in the other failure tests a copy is never issued, and nothing invalid is."""
import pytest
import torch

from paper_2608_26574_gb300 import binding as B

from .test_gpu_mlp import _check_experts, _experts_case, _run_experts

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("mx", [True, False])
@pytest.mark.parametrize("drop", [0, 2, 5, 6, 9])
def test_pairs_leave_together(monkeypatch, mx, drop):
    """A copy of a later turn of the six stages, of a second tile, and of phase 2 alone."""
    t, n, k, d, f = 900, 12, 2, 512, 2048
    c = _experts_case(t, n, k, d, f, mx, 51)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    with monkeypatch.context() as m:
        m.setenv("DARD_TEST_WAIT_CYCLES", str(1 << 20))
        m.setenv("DARD_TEST_DROP_KV", str(drop))
        _run_experts(c, n, mx, status=status)
    assert int(status.item()) == B.STATUS_TIMEOUT
    status.zero_()
    got = _run_experts(c, n, mx, status=status)
    assert int(status.item()) == 0
    some = dict(c, **{name: c[name][:50] for name in ("x", "ids", "weights")})
    _check_experts(some, got[:50], mx)
