"""Waits of the shared-prefix attention that run out at other places than in test_gpu_prefix_failure.py: a copy that
is never issued, at the first, a middle and the last tile of the prefix and at the sequences' own, in one part
or in several. The launch ends with its status bit, and the next call is right."""
import pytest
import torch

from paper_2608_26574_gb300 import binding as B

from . import test_gpu_prefix as T

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("seqs,prefix,drops", [([(3, 16, 2, 16), (0, 8, 0, 8)], 500, (0, 2, 3, 4)),
                                               ([(200, 30, 9, 30)] * 2, 140, (1, 2, 3, 5)),
                                               ([(1, 0, 0, 0)], 4096, (0,))])
@pytest.mark.parametrize("ws", [True, False])
def test_attention_wait_runs_out_anywhere(monkeypatch, d, seqs, prefix, drops, ws):
    lays, t = T.make("bf16", 8, 2, d, prefix, seqs, 7)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    for drop in drops:
        monkeypatch.setenv("DARD_TEST_WAIT_CYCLES", str(1 << 20))  # about half a millisecond
        monkeypatch.setenv("DARD_TEST_DROP_KV", str(drop))
        T.attend(lays, t, ws=ws, status=status)
        if not ws:  # (a part of a split may have fewer tiles)
            assert status.item() & B.STATUS_TIMEOUT
        monkeypatch.delenv("DARD_TEST_WAIT_CYCLES")
        monkeypatch.delenv("DARD_TEST_DROP_KV")
        status.zero_()
        T.check_attention(lays, t, *T.attend(lays, t, ws=ws, status=status))
        assert status.item() == 0
