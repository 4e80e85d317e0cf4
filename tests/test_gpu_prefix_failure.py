"""Failure paths of the shared-prefix calls, without a GPU fault (see test_gpu_failure.py): a copy
that is never issued makes every wait behind it run out, the launch ends with a status bit, and the
next call is right; a launch that the host reports as failed is an error, and the next call works."""
import pytest
import torch

from paper_2608_26574_gb300 import binding as B

from . import test_gpu_prefix as T

pytestmark = pytest.mark.gpu
DEV = "cuda"


def _attention(prefix, ws):
    lays, t = T.make("bf16", 8, 2, 128, prefix, [(3, 16, 2, 16), (0, 8, 0, 8)], 7)
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    return lays, t, status, lambda: T.attend(lays, t, ws=ws, status=status)


@pytest.mark.parametrize("prefix,ws", [(400, False), (4000, True)])
def test_attention_wait_runs_out(monkeypatch, prefix, ws):
    lays, t, status, run = _attention(prefix, ws)
    monkeypatch.setenv("DARD_TEST_WAIT_CYCLES", str(1 << 20))  # about half a millisecond
    monkeypatch.setenv("DARD_TEST_DROP_KV", "0" if ws else "1")
    run()
    assert status.item() & B.STATUS_TIMEOUT
    monkeypatch.delenv("DARD_TEST_WAIT_CYCLES")
    monkeypatch.delenv("DARD_TEST_DROP_KV")
    status.zero_()
    T.check_attention(lays, t, *run())
    assert status.item() == 0


@pytest.mark.parametrize("drop", ["0", "1", "7"])
def test_weights_wait_runs_out(monkeypatch, drop):
    _, t = T.make("bf16", 8, 2, 64, 300, [(600, 0, 0, 0)], 7)
    lse = torch.full((600, 8), 7.0, device=DEV)
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    w = torch.zeros(2, 300, device=DEV)
    monkeypatch.setenv("DARD_TEST_WAIT_CYCLES", str(1 << 20))
    monkeypatch.setenv("DARD_TEST_DROP_KV", drop)
    B.dard_prefix_weights(t["q"], lse, t["pk"], w, status=status)
    torch.cuda.synchronize()
    assert status.item() == B.STATUS_TIMEOUT
    monkeypatch.delenv("DARD_TEST_WAIT_CYCLES")
    monkeypatch.delenv("DARD_TEST_DROP_KV")
    status.zero_()
    B.dard_prefix_weights(t["q"], lse, t["pk"], w, status=status)
    torch.cuda.synchronize()
    T.check_weights(t["q"], lse, t["pk"], w)
    assert status.item() == 0


@pytest.mark.parametrize("which", ["attention", "weights", "evict"])
def test_injected_launch_failure(monkeypatch, which):
    lays, t, _, attention = _attention(100, True)
    w = torch.rand(2, 100, device=DEV)
    run = {"attention": attention,
           "weights": lambda: T.weigh(t["q"], torch.zeros(t["q"].shape[:2], device=DEV), t["pk"]),
           "evict": lambda: T.evict(w, t["pk"], t["pv"], 30)}[which]
    monkeypatch.setenv("DARD_TEST_FAIL_LAUNCH", "1")
    with pytest.raises(B.DardError) as err:
        run()
    assert err.value.code == 5 and "DARD_TEST_FAIL_LAUNCH" in str(err.value)
    monkeypatch.delenv("DARD_TEST_FAIL_LAUNCH")
    run()
