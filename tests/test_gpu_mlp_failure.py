"""Failure paths of the experts' MLP operators, exercised without a GPU fault.

A wait that runs out: with a short wait bound (DARD_TEST_WAIT_CYCLES) the products of dard_experts
are told never to issue one stage's weight copy (DARD_TEST_DROP_KV; nothing invalid is issued,
the copy simply never lands). Every wait that depends on it gives up, the launches end with
DARD_STATUS_TIMEOUT in the status word, and a normal call afterwards is right. An injected launch
failure (DARD_TEST_FAIL_LAUNCH) returns DARD_ERR_CUDA without a launch, and the next call works.
"""
import pytest
import torch

from paper_2608_26574_gb300 import binding as B

from .test_gpu_mlp import _check_experts, _experts_case, _run_experts

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("mx", [True, False])
@pytest.mark.parametrize("t,n,k,d,f", [
    (5, 4, 2, 512, 512),       # few tokens: two launches, the last tile adds the slots
    (90, 2, 1, 512, 512),      # single CTAs, y written by the product
    (900, 12, 2, 512, 1024)])  # pairs of CTAs
def test_wait_runs_out_and_the_device_stays_usable(monkeypatch, mx, t, n, k, d, f):
    c = _experts_case(t, n, k, d, f, mx, t)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    monkeypatch.setenv("DARD_TEST_WAIT_CYCLES", str(1 << 20))  # about half a millisecond
    monkeypatch.setenv("DARD_TEST_DROP_KV", "1")
    _run_experts(c, n, mx, status=status)
    assert int(status.item()) & B.STATUS_TIMEOUT
    monkeypatch.delenv("DARD_TEST_WAIT_CYCLES")
    monkeypatch.delenv("DARD_TEST_DROP_KV")
    status.zero_()
    got = _run_experts(c, n, mx, status=status)
    assert int(status.item()) == 0
    some = dict(c, **{m: c[m][:60] for m in ("x", "ids", "weights")})
    _check_experts(some, got[:60], mx)


def test_injected_launch_failure(monkeypatch):
    x = torch.randn(8, 64, device="cuda")
    codes = torch.empty(8, 64, dtype=torch.uint8, device="cuda")
    scales = torch.empty(B.mx_scale_shape((8, 64)), dtype=torch.uint8, device="cuda")
    ids = torch.empty(8, 2, dtype=torch.int32, device="cuda")
    weights = torch.empty(8, 2, device="cuda")
    c = _experts_case(6, 3, 2, 64, 64, True, 1)
    y = torch.empty_like(x)
    calls = [lambda: B.dard_residual_norm(x, y=y),
             lambda: B.dard_mx_quantize(x, codes, scales),
             lambda: B.dard_route(x, ids, weights, 2),
             lambda: _run_experts(c, 3, True)]
    for call in calls:
        monkeypatch.setenv("DARD_TEST_FAIL_LAUNCH", "1")
        with pytest.raises(B.DardError) as err:
            call()
        assert err.value.code == 5 and "launch failed" in str(err.value)  # DARD_ERR_CUDA
        monkeypatch.delenv("DARD_TEST_FAIL_LAUNCH")
        call()
    torch.cuda.synchronize()
    assert torch.isfinite(y).all()
