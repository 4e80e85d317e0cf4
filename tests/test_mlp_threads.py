"""Prepared calls of the experts' MLP shared by threads: each launch gets its own call's arguments,
whatever another thread does meanwhile. Runs on the host: the library's functions are stand-ins that
look at their arguments, wait without the interpreter lock as a library call does, and look
again; the tensors are descriptions of device tensors."""
import ctypes
import itertools
import threading
import time

import pytest
import torch

from paper_2608_26574_gb300 import binding as B
from paper_2608_26574_gb300 import build as BUILD


class Device:
    """A contiguous tensor on device 0, as far as the binding looks at it."""
    is_cuda = True
    pointers = itertools.count(0x10000, 0x10000)

    def __init__(self, *shape, dtype=torch.float32):
        self.shape, self.dtype = torch.Size(shape), dtype
        self.ptr = next(Device.pointers)

    def get_device(self):
        return 0

    def dim(self):
        return len(self.shape)

    def numel(self):
        return self.shape.numel()

    def element_size(self):
        return self.dtype.itemsize

    def is_contiguous(self):
        return True

    def data_ptr(self):
        return self.ptr

    def stride(self):
        s = [1]
        for n in self.shape[:0:-1]:
            s.insert(0, s[0] * n)
        return tuple(s)


def _norm():
    call = B.NormCall(64, torch.float32)
    return (call, B.NormArgs, lambda: (Device(3, 64), None, Device(3, 64), Device(3, 64)),
            ("x", "residual", "y"))


def _route():
    call = B.RouteCall(16, 2)

    def args():
        return Device(5, 16), Device(5, 2, dtype=torch.int32), Device(5, 2)
    return call, B.RouteArgs, args, ("logits", "ids", "weights")


def _experts():
    w = [Device(4, 96, 64, dtype=torch.bfloat16), Device(4, 96, 64, dtype=torch.bfloat16),
         Device(4, 64, 96, dtype=torch.bfloat16)]
    call = B.ExpertsCall(w[0], None, w[1], None, w[2], None, Device(1 << 20, dtype=torch.uint8))

    def args():
        i32 = torch.int32
        return (Device(6, 64, dtype=torch.bfloat16), None, Device(6, 2, dtype=i32), Device(6, 2),
                Device(5, dtype=i32), Device(12, dtype=i32), Device(6, 64, dtype=torch.bfloat16))
    return call, B.ExpertsArgs, args, ("x", "ids", "weights", "offsets", "rows", "y")


@pytest.mark.parametrize("make", [_norm, _route, _experts])
def test_threads_share_a_call(make):
    BUILD.build()
    call, struct, args, names = make()
    assert call.layout.size == ctypes.sizeof(struct)
    wanted, wrong = {}, []

    def library(packed, stream):
        want = wanted[threading.get_ident()]
        for _ in range(2):
            a = struct.from_buffer_copy(packed)
            got = tuple(getattr(a, n) for n in names)
            if got != want:
                wrong.append((got, want))
            time.sleep(0.0005)
        return 0

    call._fn = library

    def work():
        for _ in range(40):
            a = args()
            wanted[threading.get_ident()] = tuple(t.ptr for t in a if t is not None)
            call(*a, stream=1)

    threads = [threading.Thread(target=work) for _ in range(4)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not wrong
