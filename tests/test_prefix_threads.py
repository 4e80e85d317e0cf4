"""Prepared calls of the shared prefix shared by threads: each launch gets its own call's arguments.
Runs on the host, with stand-ins for the tensors and the library (see test_mlp_threads.py)."""
import ctypes
import threading
import time

import pytest
import torch

from paper_2608_26574_gb300 import binding as B
from paper_2608_26574_gb300 import build as BUILD

from .test_mlp_threads import Device

BF = torch.bfloat16


def _attention():
    call = B.PrefixAttentionCall([3], [0], [0], [0], None, None, None)
    return call, B.PrefixAttnArgs, lambda: (
        Device(3, 4, 64, dtype=BF), Device(3, 2, 64, dtype=BF), Device(3, 2, 64, dtype=BF),
        Device(3, 4, 64, dtype=BF), Device(9, 2, 64, dtype=BF), Device(9, 2, 64, dtype=BF)), \
        lambda a: (a.own.q, a.own.k, a.own.v, a.own.o, a.prefix_k, a.prefix_v)


def _weights():
    call = B.PrefixWeightsCall()
    return call, B.PrefixWeightsArgs, lambda: (
        Device(3, 4, 64, dtype=BF), Device(3, 4), Device(9, 2, 64, dtype=BF), Device(2, 9)), \
        lambda a: (a.q, a.lse, a.prefix_k, a.weights)


def _evict():
    call = B.PrefixEvictCall(1, 1)
    return call, B.PrefixEvictArgs, lambda: (
        Device(2, 9), Device(9, 2, 64, dtype=BF), Device(9, 2, 64, dtype=BF),
        Device(2, 5, dtype=torch.int32), Device(5, 2, 64, dtype=BF), Device(5, 2, 64, dtype=BF)), \
        lambda a: (a.weights, a.prefix_k, a.prefix_v, a.kept, a.k_out, a.v_out)


@pytest.mark.parametrize("make", [_attention, _weights, _evict])
def test_calls_shared_by_threads(make, monkeypatch):
    BUILD.build()
    B.lib()
    monkeypatch.setattr(B, "_current_device", lambda: 0)
    monkeypatch.setattr(B, "_raw_stream", lambda i: 0)
    call, struct, args, fields = make()
    seen, wrong = [], []

    def library(packed, stream):
        a = struct.from_buffer_copy(packed)
        first = fields(a)
        time.sleep(0.002)  # (without the interpreter lock, as a library call is)
        again = fields(struct.from_buffer_copy(packed))
        if again != first:
            wrong.append((first, again))
        seen.append(first)
        return 0

    call._fn = library
    expected, lock = [], threading.Lock()

    def run():
        for _ in range(10):
            t = args()
            with lock:
                expected.append(tuple(x.ptr for x in t))
            call(*t)

    threads = [threading.Thread(target=run) for _ in range(4)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not wrong and sorted(seen) == sorted(expected)


def test_launch_on_another_device(monkeypatch):
    """A call on tensors of another device than the current one makes that device current for it."""
    entered = []

    class Guard:
        def __init__(self, d):
            self.d = d

        def __enter__(self):
            entered.append(self.d)

        def __exit__(self, *a):
            entered.append(None)

    BUILD.build()
    B.lib()
    monkeypatch.setattr(B, "_current_device", lambda: 1)
    monkeypatch.setattr(torch.cuda, "device", Guard)
    monkeypatch.setattr(B, "_raw_stream", lambda i: 100 + i)
    calls = []
    B._launch(lambda a, s: calls.append((a, s, list(entered))) or 0, "f", b"x", None, 0)
    assert calls == [(b"x", 100, [0])] and entered == [0, None]
    assert ctypes.sizeof(B.PrefixEvictArgs) == 128
