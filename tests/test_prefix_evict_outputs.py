"""Outputs of dard_prefix_evict that share memory with one another or with themselves are refused, and only
those, against brute force over the bytes (on the host, before any launch: the pointers are never followed)."""
import ctypes
import itertools
import random

import pytest

from paper_2608_26574_gb300 import binding as B
from paper_2608_26574_gb300 import build as BUILD

VALUE = 3
BASE = 1 << 40


@pytest.fixture(scope="module")
def lib():
    BUILD.build()
    return B.lib()


def _args(keep, hkv, d, dtype, row, head, k_out, v_out, kept, weights_out):
    a = B.PrefixEvictArgs()
    a.weights, a.prefix_k, a.prefix_v = 1 << 30, 1 << 31, 1 << 32
    a.kept, a.k_out, a.v_out, a.weights_out = kept, k_out, v_out, weights_out
    a.weights_stride, a.prefix_row_stride, a.prefix_head_stride = 100, hkv * d, d
    a.out_row_stride, a.out_head_stride = row, head
    a.dtype, a.hkv, a.head_dim, a.prefix_len, a.keep = dtype, hkv, d, 100, keep
    return a


def _refused(lib, a, monkeypatch):
    """Whether the outputs are refused; a call whose arguments are in order comes to its (injected) launch."""
    monkeypatch.setenv("DARD_TEST_FAIL_LAUNCH", "1")
    code = lib.dard_prefix_evict(ctypes.byref(a), None)
    assert code in (VALUE, 5), lib.dard_last_error()
    if code == VALUE:
        assert b"overlap" in lib.dard_last_error()
    return code == VALUE


def _blocks(base, keep, hkv, row, head, run):
    return [(base + r * row + g * head, run) for r in range(keep) for g in range(hkv)]


def _overlap(blocks):
    blocks = sorted(blocks)
    return any(a + n > b for (a, n), (b, _) in itertools.pairwise(blocks))


@pytest.mark.parametrize("keep,row,head,refused", [
    (40, 256, 128, False), (40, 128, 128 * 40, False), (40, 128, 128, True), (1, 128, 128, False),
    (40, 256, 384, False), (40, 256, 320, True), (40, 256, 256, True), (40, 384, 128, False), (40, 136, 128, True), (3, 128, 384, False),
    (4, 128, 384, True), (40, 1 << 36, 1 << 36, True), (40, 1 << 36, 1 << 35, False)])
def test_strides_that_collide(lib, monkeypatch, keep, row, head, refused):
    """Rows of two heads of 128 elements."""
    a = _args(keep, 2, 128, B.DARD_BF16, row, head, BASE, 1 << 55, 1 << 33, 1 << 34)
    assert _refused(lib, a, monkeypatch) == refused


def test_outputs_in_one_another(lib, monkeypatch):
    ok = dict(keep=40, hkv=2, d=128, dtype=B.DARD_BF16, row=256, head=128, k_out=BASE, v_out=BASE + 40 * 512,
              kept=1 << 33, weights_out=1 << 34)
    assert not _refused(lib, _args(**ok), monkeypatch)
    # keys and values row by row, and head by head, beside each other
    assert not _refused(lib, _args(**{**ok, "row": 512, "v_out": BASE + 512}), monkeypatch)
    assert not _refused(lib, _args(**{**ok, "row": 512, "head": 256, "v_out": BASE + 256}), monkeypatch)
    for change in ({"v_out": BASE}, {"v_out": BASE + 39 * 512}, {"v_out": BASE + 16}, {"kept": BASE},
                   {"kept": BASE - 4}, {"weights_out": BASE + 40 * 512 - 4}, {"weights_out": (1 << 33) + 4 * 79},
                   {"kept": BASE + 40 * 1024 - 320 + 4, "v_out": BASE + 40 * 512}):
        assert _refused(lib, _args(**{**ok, **change}), monkeypatch), change
    # without keys and values the lists are looked at all the same
    a = _args(**{**ok, "weights_out": 1 << 33})
    a.prefix_k = a.prefix_v = a.k_out = a.v_out = None
    assert _refused(lib, a, monkeypatch)
    a.weights_out = None
    assert not _refused(lib, a, monkeypatch)


def test_outputs_against_brute_force(lib, monkeypatch):
    rng = random.Random(5)
    seen = set()
    for _ in range(4000):
        keep, hkv, esz = rng.randint(1, 6), rng.randint(1, 4), rng.choice([2, 4])
        unit = 16 // esz
        row, head = (64 + unit * rng.choice([0, 0, 1, 8, rng.randint(0, 60)]) + 64 * rng.randint(0, 8) for _ in range(2))
        k = BASE
        v = BASE + 16 * rng.randint(-400, 400)
        kept = BASE + 4 * rng.randint(-1200, 1200) if rng.random() < 0.5 else 1 << 33
        w = BASE + 4 * rng.randint(-1200, 1200) if rng.random() < 0.5 else 1 << 34
        a = _args(keep, hkv, 64, B.DARD_BF16 if esz == 2 else B.DARD_F32, row, head, k, v, kept, w)
        blocks = [b for base in (k, v) for b in _blocks(base, keep, hkv, row * esz, head * esz, 64 * esz)]
        want = _overlap(blocks + [(kept, 4 * keep * hkv), (w, 4 * keep * hkv)])
        assert _refused(lib, a, monkeypatch) == want, (keep, hkv, esz, row, head, v - k, kept - k, w - k)
        seen.add(want)
    assert seen == {True, False}


def test_tensors_beyond_any_address(lib, monkeypatch):
    """Rows times strides that pass 64 bits would meet nothing, or anything."""
    for change in ({"keep": 1 << 30, "out_row_stride": 1 << 36}, {"prefix_row_stride": 1 << 36},
                   {"weights_stride": 1 << 62}):
        a = _args(40, 2, 128, B.DARD_BF16, 256, 128, BASE, 1 << 55, 1 << 33, 1 << 34)
        a.prefix_len = a.weights_stride = 1 << 30
        for k, v in change.items():
            setattr(a, k, v)
        monkeypatch.setenv("DARD_TEST_FAIL_LAUNCH", "1")
        assert lib.dard_prefix_evict(ctypes.byref(a), None) == 2
        assert b"2^60" in lib.dard_last_error()
