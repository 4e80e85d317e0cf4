"""Refusals of the shared-prefix entry points: every argument that the library or the binding turns
down, on the host, before any launch (no GPU needed: the pointers are never followed)."""
import ctypes

import numpy as np
import pytest
import torch

from oracle import prefix_oracle as O
from paper_2608_26574_gb300 import binding as B
from paper_2608_26574_gb300 import build as BUILD

NULL, SHAPE, VALUE, UNSUPPORTED, CUDA, ALIGN, WORKSPACE = 1, 2, 3, 4, 5, 6, 7
PTR = 0x100000


@pytest.fixture(scope="module")
def lib():
    BUILD.build()
    return B.lib()


def _refuse(lib, fn, args, change, code):
    for k, v in change.items():
        tgt = args
        if k.startswith("own."):
            tgt, k = args.own, k[4:]
        setattr(tgt, k, v)
    assert getattr(lib, fn)(ctypes.byref(args), None) == code
    assert lib.dard_last_error().decode() != ""


_HOLD = []


def _i32(*v):
    a = (ctypes.c_int32 * len(v))(*v)
    _HOLD.append(a)
    return ctypes.cast(a, ctypes.POINTER(ctypes.c_int32))


def _attn():
    a = B.PrefixAttnArgs()
    o = a.own
    o.q, o.k, o.v, o.o = PTR, 2 * PTR, 3 * PTR, 4 * PTR
    o.dtype, o.hq, o.hkv, o.head_dim, o.num_seqs = B.DARD_BF16, 8, 2, 128, 2
    o.n_orig, o.block_start, o.block_len, o.shadow_len = _i32(5, 9), _i32(1, 0), _i32(4, 0), _i32(4, 0)
    o.state, o.prev_conf, o.shadow_src = PTR, PTR, PTR
    a.prefix_k, a.prefix_v = 5 * PTR, 6 * PTR
    a.prefix_row_stride, a.prefix_head_stride, a.prefix_len = 256, 128, 1000
    return a


@pytest.mark.parametrize("fn", ["dard_prefix_attention", "dard_prefix_weights", "dard_prefix_evict"])
def test_null_args(lib, fn):
    assert getattr(lib, fn)(None, None) == NULL


@pytest.mark.parametrize("change,code", [
    ({"own.q": None}, NULL), ({"own.o": None}, NULL), ({"own.n_orig": None}, NULL),
    ({"own.state": None}, NULL), ({"own.shadow_src": None}, NULL), ({"own.num_seqs": 0}, SHAPE),
    ({"own.num_seqs": 257}, SHAPE), ({"own.hq": 7}, SHAPE), ({"own.head_dim": 96}, UNSUPPORTED),
    ({"own.dtype": 2}, VALUE), ({"own.scale": -1.0}, VALUE), ({"own.scale": float("nan")}, VALUE),
    ({"own.rope_theta": 10000.0, "own.k_rope": PTR}, VALUE), ({"own.q": PTR + 8}, ALIGN),
    ({"own.n_orig": _i32(0, 9)}, SHAPE), ({"own.block_start": _i32(2, 0)}, SHAPE),
    ({"own.query_start": _i32(10, 0)}, SHAPE),
    ({"prefix_k": None}, NULL), ({"prefix_v": None}, NULL), ({"prefix_len": -1}, SHAPE),
    ({"prefix_len": B.PREFIX_MAX_LEN + 1}, SHAPE), ({"prefix_row_stride": 64}, SHAPE),
    ({"prefix_row_stride": -256}, SHAPE), ({"prefix_head_stride": 0}, SHAPE),
    ({"prefix_head_stride": 1 << 37}, SHAPE), ({"prefix_row_stride": 257}, ALIGN),
    ({"prefix_head_stride": 132}, ALIGN), ({"prefix_k": 5 * PTR + 8}, ALIGN),
    ({"prefix_v": 5 * PTR + 2}, ALIGN), ({"lse": PTR + 2}, ALIGN),
    ({"workspace": PTR, "workspace_bytes": 1000}, WORKSPACE),
    ({"workspace": PTR + 8, "workspace_bytes": 1 << 40}, ALIGN)])
def test_attention_refusals(lib, change, code):
    _refuse(lib, "dard_prefix_attention", _attn(), change, code)


def test_attention_too_many_queries(lib):
    """Rows times the heads of a group stay below 2^31."""
    a = _attn()
    a.own.num_seqs = 1
    a.own.n_orig, a.own.block_start = _i32(1 << 30), _i32(0)
    a.own.block_len, a.own.shadow_len = _i32(0), _i32(0)
    a.own.hq, a.own.hkv, a.own.head_dim = 8, 1, 64
    _refuse(lib, "dard_prefix_attention", a, {}, SHAPE)


def _weights():
    a = B.PrefixWeightsArgs()
    a.q, a.lse, a.prefix_k, a.weights = PTR, 2 * PTR, 3 * PTR, 4 * PTR
    a.prefix_row_stride, a.prefix_head_stride, a.weights_stride = 256, 128, 100
    a.dtype, a.rows, a.hq, a.hkv, a.head_dim, a.prefix_len, a.decay = B.DARD_BF16, 5, 8, 2, 128, 100, 1.0
    return a


@pytest.mark.parametrize("change,code", [
    ({"q": None}, NULL), ({"lse": None}, NULL), ({"prefix_k": None}, NULL), ({"weights": None}, NULL),
    ({"dtype": 2}, VALUE), ({"rows": -1}, SHAPE), ({"hq": 7}, SHAPE), ({"hkv": 0}, SHAPE),
    ({"hq": 1 << 17, "hkv": 1 << 17}, SHAPE), ({"rows": 1 << 30}, SHAPE), ({"head_dim": 32}, UNSUPPORTED),
    ({"prefix_len": -1}, SHAPE), ({"prefix_len": B.PREFIX_MAX_LEN + 1}, SHAPE), ({"scale": -0.5}, VALUE),
    ({"scale": float("inf")}, VALUE), ({"decay": float("nan")}, VALUE), ({"weights_stride": 99}, SHAPE),
    ({"weights_in": PTR, "weights_in_stride": 10}, SHAPE),
    ({"weights_in": 4 * PTR, "weights_in_stride": 200}, VALUE), ({"weights": PTR + 2}, ALIGN),
    ({"lse": PTR + 1}, ALIGN), ({"q": PTR + 8}, ALIGN), ({"prefix_row_stride": 127}, SHAPE),
    ({"prefix_row_stride": 260}, ALIGN), ({"prefix_k": PTR + 2}, ALIGN),
    ({"workspace": PTR, "workspace_bytes": 16}, WORKSPACE),
    ({"workspace": PTR + 4, "workspace_bytes": 1 << 40}, ALIGN)])
def test_weights_refusals(lib, change, code):
    _refuse(lib, "dard_prefix_weights", _weights(), change, code)


@pytest.mark.parametrize("at,stride,in_stride,hkv,refused", [
    # weights [2, 100] at 4 PTR, 100 or 250 elements between heads; the earlier sums `at` elements on
    (1, 100, 100, 2, True), (199, 100, 100, 2, True), (200, 100, 100, 2, False), (-199, 100, 100, 2, True),
    (-200, 100, 100, 2, False), (100, 250, 250, 2, False), (150, 250, 250, 2, False), (99, 250, 250, 2, True),
    (151, 250, 250, 2, True), (-100, 250, 250, 2, False), (-99, 250, 250, 2, True), (400, 250, 250, 2, False),
    (300, 250, 120, 2, True), (350, 250, 120, 2, False), (50, 100, 100, 1, True), (100, 100, 100, 1, False)])
def test_weights_beside_their_earlier_sums(lib, at, stride, in_stride, hkv, refused):
    """weights_in is weights itself or has no element in common with it. (The calls that are not refused
    for that end with a launch that fails, as there is no device here, or with the workspace's size.)"""
    a = _weights()
    a.hkv, a.weights_stride, a.weights_in_stride, a.weights_in = hkv, stride, in_stride, 4 * PTR + 4 * at
    _refuse(lib, "dard_prefix_weights", a, {"workspace": 9 * PTR, "workspace_bytes": 16},
            VALUE if refused else WORKSPACE)


def _evict():
    a = B.PrefixEvictArgs()
    a.weights, a.prefix_k, a.prefix_v, a.kept, a.k_out, a.v_out = (i * PTR for i in range(1, 7))
    a.weights_stride, a.prefix_row_stride, a.prefix_head_stride = 100, 256, 128
    a.out_row_stride, a.out_head_stride = 256, 128
    a.dtype, a.hkv, a.head_dim, a.prefix_len, a.keep, a.keep_first, a.keep_last = B.DARD_BF16, 2, 128, 100, 40, 4, 8
    return a


@pytest.mark.parametrize("change,code", [
    ({"weights": None}, NULL), ({"kept": None}, NULL), ({"prefix_k": None}, NULL), ({"v_out": None}, NULL),
    ({"dtype": 3}, VALUE), ({"hkv": 0}, SHAPE), ({"hkv": 65536}, SHAPE), ({"head_dim": 256}, UNSUPPORTED),
    ({"prefix_len": -1}, SHAPE), ({"keep": 101}, SHAPE), ({"keep": -1}, SHAPE), ({"keep": 11}, SHAPE),
    ({"keep_first": -1}, SHAPE), ({"keep_last": -1}, SHAPE),
    ({"keep_first": (1 << 31) - 1, "keep_last": (1 << 31) - 1}, SHAPE), ({"weights_stride": 99}, SHAPE),
    ({"prefix_row_stride": 100}, SHAPE), ({"out_head_stride": 64}, SHAPE), ({"out_row_stride": 257}, ALIGN),
    ({"k_out": 5 * PTR + 8}, ALIGN), ({"weights_out": PTR * 7 + 2}, ALIGN), ({"kept": PTR * 4 + 1}, ALIGN),
    # outputs over inputs: in place, at the last byte, and the lists over the weights
    ({"k_out": 2 * PTR}, VALUE), ({"v_out": 2 * PTR + 99 * 512 + 240 + 256}, VALUE),
    ({"kept": PTR + 792}, VALUE), ({"weights_out": PTR}, VALUE)])
def test_evict_refusals(lib, change, code):
    _refuse(lib, "dard_prefix_evict", _evict(), change, code)


def test_nothing_to_do_is_no_error(lib):
    """No query rows, no prefix, nothing to keep: success without a launch (there is no device here)."""
    a = _attn()
    a.own.query_start = _i32(9, 9)
    assert lib.dard_prefix_attention(ctypes.byref(a), None) == 0
    a = _weights()
    a.prefix_len, a.q, a.weights = 0, None, None
    assert lib.dard_prefix_weights(ctypes.byref(a), None) == 0
    a = _evict()
    a.keep = a.keep_first = a.keep_last = 0
    a.kept = None
    assert lib.dard_prefix_evict(ctypes.byref(a), None) == 0


def test_workspace_sizes(lib):
    """Enough for smaller calls, 0 for invalid sizes."""
    for f in (B.dard_prefix_attention_workspace_size, B.dard_prefix_weights_workspace_size):
        big = f(5000, 32, 8, 128, 100000)
        assert big > 0
        for rows, hq, hkv, d, n in ((1, 32, 8, 128, 100000), (5000, 8, 8, 128, 1), (5000, 32, 8, 64, 100000)):
            assert 0 < f(rows, hq, hkv, d, n) <= big
        assert f(1, 7, 2, 128, 5) == 0 and f(-1, 8, 2, 128, 5) == 0 and f(1, 8, 2, 96, 5) == 0
        assert f(1, 8, 2, 128, -1) == 0


def test_struct_layouts():
    """The packed layouts of the calls are those of the C structs."""
    for call, args in ((B.PrefixAttentionCall, B.PrefixAttnArgs), (B.PrefixWeightsCall, B.PrefixWeightsArgs),
                       (B.PrefixEvictCall, B.PrefixEvictArgs)):
        assert call.layout.size == ctypes.sizeof(args)
    n = len(B.PrefixEvictArgs._fields_)
    got = B.PrefixEvictArgs.from_buffer_copy(B.PrefixEvictCall.layout.pack(*range(1, n + 1)))
    assert [getattr(got, f[0]) for f in B.PrefixEvictArgs._fields_] == list(range(1, n + 1))
    n = len(B.PrefixWeightsArgs._fields_)
    got = B.PrefixWeightsArgs.from_buffer_copy(B.PrefixWeightsCall.layout.pack(*range(1, n + 1)))
    assert [getattr(got, f[0]) for f in B.PrefixWeightsArgs._fields_] == list(range(1, n + 1))
    own = len(B.AttnArgs._fields_)
    got = B.PrefixAttnArgs.from_buffer_copy(B.PrefixAttentionCall.layout.pack(*range(1, own + 9)))
    for i, (name, kind) in enumerate(B.AttnArgs._fields_):
        value = getattr(got.own, name)
        if kind is B._I32P:
            value = ctypes.cast(value, ctypes.c_void_p).value
        assert value == i + 1, name
    for i, (name, _) in enumerate(B.PrefixAttnArgs._fields_[1:]):
        assert getattr(got, name) == own + i + 1, name


def test_binding_refuses_before_the_library(lib):
    """Host tensors, wrong types, shapes and devices raise ValueError in the binding."""
    bf, f32 = torch.bfloat16, torch.float32
    q, kv = torch.zeros(6, 4, 64, dtype=bf), torch.zeros(6, 2, 64, dtype=bf)
    call = B.PrefixAttentionCall([6], [0], [0], [0], None, None, None)
    with pytest.raises(ValueError, match="device tensor"):
        call(q, kv, kv, q, kv, kv)
    with pytest.raises(ValueError, match="expected, got"):
        call(q[:5], kv, kv, q[:5], kv, kv)
    with pytest.raises(ValueError, match="differ in length"):
        B.PrefixAttentionCall([6, 1], [0], [0], [0], None, None, None)
    with pytest.raises(ValueError, match="device tensor"):
        B.PrefixAttentionCall([6], [0], [4], [0], torch.zeros(4, dtype=torch.uint8), None, None)
    with pytest.raises(ValueError, match="device tensor"):
        B.PrefixWeightsCall()(q, torch.zeros(6, 4), kv, torch.zeros(2, 6))
    with pytest.raises(ValueError, match="device tensor"):
        B.dard_prefix_evict(torch.zeros(2, 6), kv, kv, None, kv, kv)
    with pytest.raises(ValueError, match="prefix_k"):
        B._cache(kv.to(f32), "prefix_k", -1, bf, 2, 64)


def test_strides_that_no_step_uses(lib):
    """Rows of an empty or one-row cache, heads of a one-head cache: any stride will do."""
    class Fake:
        dtype = torch.bfloat16

        def __init__(self, shape, strides):
            self.shape, self.strides = torch.Size(shape), strides

        def get_device(self):
            return 0

        def stride(self):
            return self.strides

        def data_ptr(self):
            return PTR

    def strides(shape, s):
        return B._cache(Fake(shape, s), "k", 0, torch.bfloat16, shape[1], 64)[1:]

    assert strides((0, 2, 64), (1, 3, 1)) == (128, 64)
    assert strides((1, 2, 64), (1, 72, 1)) == (128, 72)
    assert strides((9, 1, 64), (80, 0, 1)) == (80, 64)
    for shape, s in (((9, 2, 64), (128, 8, 1)), ((9, 2, 64), (32, 64, 1)), ((9, 2, 64), (128, 64, 2))):
        with pytest.raises(ValueError):
            strides(shape, s)


def test_prefix_cache_refusals(lib):
    from paper_2608_26574_gb300.prefix import PrefixCache
    with pytest.raises(ValueError, match="CUDA device"):
        PrefixCache(1, 4, 2, 64, 10, device="cpu")
    with pytest.raises(ValueError, match="heads"):
        PrefixCache(1, 5, 2, 64, 10)


# ------------------------------------------------------------------ the oracle itself
def test_oracle_weights_are_the_attentions_probabilities():
    """Over the whole prefix and a query's own keys the probabilities add up to 1, and the weights
    are their sums over the prefix's keys."""
    from oracle import dard_oracle as D
    rng = np.random.default_rng(0)
    lay = [D.SeqLayout(3, 3, np.zeros(0, np.uint8), np.zeros(0, np.float32), np.zeros(0, np.int32))]
    q, k, v = (rng.normal(size=(3, 2, 8)) for _ in range(3))
    pk, pv = (rng.normal(size=(11, 2, 8)) for _ in range(2))
    o, lse, _, _ = O.prefix_attention(q, k, v, pk, pv, lay)
    w, _, _ = O.prefix_weights(q, lse, pk)
    for h in range(2):
        z = np.concatenate([q[:, h] @ pk[:, h].T, q[:, h] @ k[:, h].T], 1) / np.sqrt(8)
        p = np.exp(z) / np.exp(z).sum(1, keepdims=True)
        assert np.allclose(w[h], p[:, :11].sum(0))
        assert np.allclose(o[:, h], p @ np.concatenate([pv[:, h], v[:, h]]))


def test_oracle_evict_by_hand():
    w = [[5.0, 1.0, 3.0, np.nan, 3.0, -1.0, 9.0]]
    assert O.prefix_evict(w, 3).tolist() == [[0, 2, 6]]
    assert O.prefix_evict(w, 4).tolist() == [[0, 2, 4, 6]]
    assert O.prefix_evict(w, 6).tolist() == [[0, 1, 2, 4, 5, 6]]
    assert O.prefix_evict(w, 3, 0, 2).tolist() == [[0, 5, 6]]
    assert O.prefix_evict(w, 2, 2, 0).tolist() == [[0, 1]]
