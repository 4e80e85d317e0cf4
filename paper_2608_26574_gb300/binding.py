"""ctypes binding of libdard.so: argument marshalling only.

Each function takes torch CUDA tensors for device data and NumPy / Python integer
sequences for the per-sequence host metadata, fills the C argument struct declared in
``include/dard.h`` and calls the library entry point of the same name on the current torch
stream (or the given one). Every step of the computation runs in the library's CUDA
kernels; there is no fallback: a missing library raises.
"""
from __future__ import annotations

import ctypes
import os
import struct

import numpy as np

_PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_PKG, "libdard.so")

DARD_F32, DARD_BF16 = 0, 1
ORDER_CONFIDENCE, ORDER_BIDIR, ORDER_L2R, ORDER_ENTROPY, ORDER_MARGIN = 0, 1, 2, 3, 4
STATUS_BAD_STATE, STATUS_BAD_SHADOW, STATUS_INVALID_ROW, STATUS_TIMEOUT = 0x1, 0x2, 0x4, 0x8
MAX_SEQS, MAX_BLOCK = 256, 128
SCORE_NOALLOC_MAX_ROWS = 8192
DARD_MXFP8 = 2  # dard_experts only
MX_SCALE_ROWS, MX_SCALE_TILES = 0, 1
ROUTE_SOFTMAX, ROUTE_SIGMOID = 0, 1
MX_BLOCK = 32
NORM_MAX_DIM, MAX_EXPERTS, MAX_TOP_K, MAX_GROUPS = 32768, 512, 32, 32
EXPERTS_MAX_PAIRS = 1 << 24  # tokens * top_k of one dard_experts call

_I32P = ctypes.POINTER(ctypes.c_int32)


class AttnArgs(ctypes.Structure):
    _fields_ = [("q", ctypes.c_void_p), ("k", ctypes.c_void_p), ("v", ctypes.c_void_p),
                ("o", ctypes.c_void_p), ("dtype", ctypes.c_int32), ("hq", ctypes.c_int32),
                ("hkv", ctypes.c_int32), ("head_dim", ctypes.c_int32),
                ("num_seqs", ctypes.c_int32), ("n_orig", _I32P), ("block_start", _I32P),
                ("block_len", _I32P), ("shadow_len", _I32P), ("state", ctypes.c_void_p),
                ("prev_conf", ctypes.c_void_p), ("shadow_src", ctypes.c_void_p),
                ("scale", ctypes.c_float), ("status", ctypes.c_void_p),
                ("query_start", _I32P), ("rope_theta", ctypes.c_float),
                ("rope_style", ctypes.c_int32), ("k_rope", ctypes.c_void_p)]

DARD_ROPE_INTERLEAVED, DARD_ROPE_HALF = 0, 1


class ScoreArgs(ctypes.Structure):
    _fields_ = [("logits_x", ctypes.c_void_p), ("logits_s", ctypes.c_void_p),
                ("dtype", ctypes.c_int32), ("vocab", ctypes.c_int32),
                ("row_stride", ctypes.c_int64), ("num_seqs", ctypes.c_int32),
                ("block_len", _I32P), ("state_in", ctypes.c_void_p),
                ("tau_c", ctypes.c_float), ("tau_u", ctypes.c_float),
                ("lambda_", ctypes.c_float), ("p0", ctypes.c_float),
                ("conf", ctypes.c_void_p), ("token", ctypes.c_void_p),
                ("state_out", ctypes.c_void_p), ("w_out", ctypes.c_void_p),
                ("counts", ctypes.c_void_p), ("status", ctypes.c_void_p),
                ("workspace", ctypes.c_void_p), ("workspace_bytes", ctypes.c_size_t),
                ("cur_token", ctypes.c_void_p), ("p_cur", ctypes.c_void_p),
                ("tokens", ctypes.c_void_p), ("mask_token", ctypes.c_int32),
                ("entropy", ctypes.c_void_p), ("margin", ctypes.c_void_p),
                ("order_key", ctypes.c_void_p), ("order_mode", ctypes.c_int32)]


class NormArgs(ctypes.Structure):
    _fields_ = ([(n, ctypes.c_void_p) for n in ("x", "delta", "weight", "residual", "y", "y8",
                                                "y8_scale")] +
                [("dtype", ctypes.c_int32), ("dim", ctypes.c_int32), ("rows", ctypes.c_int64)] +
                [(n, ctypes.c_int64) for n in ("x_stride", "delta_stride", "residual_stride",
                                               "y_stride", "y8_stride", "y8_scale_stride")] +
                [("eps", ctypes.c_float)])


class MxArgs(ctypes.Structure):
    _fields_ = [("x", ctypes.c_void_p), ("codes", ctypes.c_void_p), ("scales", ctypes.c_void_p),
                ("dtype", ctypes.c_int32), ("layout", ctypes.c_int32),
                ("batch", ctypes.c_int32), ("cols", ctypes.c_int32), ("rows", ctypes.c_int64),
                ("x_row_stride", ctypes.c_int64), ("x_batch_stride", ctypes.c_int64),
                ("scale_stride", ctypes.c_int64)]


class RouteArgs(ctypes.Structure):
    _fields_ = ([("logits", ctypes.c_void_p), ("logits_stride", ctypes.c_int64),
                 ("bias", ctypes.c_void_p)] +
                [(n, ctypes.c_int32) for n in ("dtype", "scoring", "tokens", "experts", "top_k",
                                               "groups", "top_groups", "renormalise")] +
                [("scale", ctypes.c_float)] +
                [(n, ctypes.c_void_p) for n in ("ids", "weights", "offsets", "rows", "status",
                                                "workspace")] +
                [("workspace_bytes", ctypes.c_size_t)])


class ExpertsArgs(ctypes.Structure):
    _fields_ = ([(n, ctypes.c_void_p) for n in ("x", "x_scale", "w1", "w3", "w2", "w1_scale",
                                                "w3_scale", "w2_scale", "ids", "weights",
                                                "offsets", "rows", "y")] +
                [(n, ctypes.c_int64) for n in ("x_stride", "x_scale_stride", "y_stride")] +
                [(n, ctypes.c_int32) for n in ("dtype", "y_dtype", "tokens", "experts", "top_k",
                                               "dim", "hidden")] +
                [("workspace", ctypes.c_void_p), ("workspace_bytes", ctypes.c_size_t),
                 ("status", ctypes.c_void_p)])


class DardError(RuntimeError):
    def __init__(self, code: int, fn: str, message: str):
        super().__init__(f"{fn} failed: {status_string(code)}: {message}")
        self.code = code


_lib = None

class AttnPlan(ctypes.Structure):
    _fields_ = [("kernel", ctypes.c_int32), ("ctas", ctypes.c_int64),
                ("tile_pairs", ctypes.c_int64), ("tile_pairs_skipped", ctypes.c_int64)]


# Exported entry points: name -> (restype, argtypes)
EXPORTS = {
    "dard_attention_plan": (ctypes.c_int, [ctypes.POINTER(AttnArgs), ctypes.POINTER(AttnPlan)]),
    "dard_step_attention": (ctypes.c_int, [ctypes.POINTER(AttnArgs), ctypes.c_void_p]),
    "dard_attention_kernel": (ctypes.c_int, [ctypes.POINTER(AttnArgs),
                                             ctypes.POINTER(ctypes.c_int32)]),
    "dard_score_and_transition": (ctypes.c_int, [ctypes.POINTER(ScoreArgs), ctypes.c_void_p]),
    "dard_score_and_transition_noalloc": (ctypes.c_int, [ctypes.POINTER(ScoreArgs),
                                                         ctypes.c_void_p]),
    "dard_score_workspace_size": (ctypes.c_size_t, [ctypes.c_int32, ctypes.c_int32, ctypes.c_int32]),
    "dard_residual_norm": (ctypes.c_int, [ctypes.POINTER(NormArgs), ctypes.c_void_p]),
    "dard_mx_quantize": (ctypes.c_int, [ctypes.POINTER(MxArgs), ctypes.c_void_p]),
    "dard_route_workspace_size": (ctypes.c_size_t, [ctypes.c_int32] * 3),
    "dard_route": (ctypes.c_int, [ctypes.POINTER(RouteArgs), ctypes.c_void_p]),
    "dard_experts_workspace_size": (ctypes.c_size_t, [ctypes.c_int32] * 5),
    "dard_experts": (ctypes.c_int, [ctypes.POINTER(ExpertsArgs), ctypes.c_void_p]),
    "dard_status_string": (ctypes.c_char_p, [ctypes.c_int]),
    "dard_last_error": (ctypes.c_char_p, []),
    "dard_version": (ctypes.c_int32, []),
}


def lib(path: str | None = None) -> ctypes.CDLL:
    """Loads libdard.so once; raises if it has not been built."""
    global _lib
    if _lib is None:
        p = path or LIB_PATH
        if not os.path.exists(p):
            raise RuntimeError(f"{p} is missing: build it with paper_2608_26574_gb300.build.build()")
        L = ctypes.CDLL(p)
        for name, (res, args) in EXPORTS.items():
            fn = getattr(L, name)
            fn.restype = res
            fn.argtypes = args
        _lib = L
    return _lib


def status_string(code: int) -> str:
    return lib().dard_status_string(code).decode()


def _check(code: int, fn: str):
    if code != 0:
        raise DardError(code, fn, lib().dard_last_error().decode())


def _host_i32(a) -> np.ndarray:
    """An owned, contiguous int32 copy of a per-sequence host array."""
    return np.array(a, dtype=np.int32, copy=True).reshape(-1)


def _torch():
    import torch
    return torch


_current_stream = None


def _raw_stream(device_index: int) -> int:
    """cudaStream_t of the device's current torch stream."""
    global _current_stream
    if _current_stream is None:
        torch = _torch()
        _current_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (
            lambda i: torch.cuda.current_stream(i).cuda_stream)
    return _current_stream(device_index)


def _stream_handle(stream, device_index: int) -> int:
    """``stream`` as a raw handle: a torch stream, an int, or None for the current stream."""
    if stream is None:
        return _raw_stream(device_index)
    if isinstance(stream, int):
        return stream
    return stream.cuda_stream


def _dtype_code(t) -> int:
    torch = _torch()
    if t.dtype == torch.bfloat16:
        return DARD_BF16
    if t.dtype == torch.float32:
        return DARD_F32
    raise ValueError(f"unsupported dtype {t.dtype}")


def _dev(t, name: str, n: int, dtype, device: int | None = None) -> int | None:
    """Device pointer of an optional contiguous tensor of ``dtype`` with at least ``n``
    elements (None for a missing tensor)."""
    if t is None:
        return None
    if not t.is_cuda:
        raise ValueError(f"{name}: device tensor expected")
    if not t.is_contiguous():
        raise ValueError(f"{name}: contiguous tensor expected")
    if t.dtype != dtype:
        raise ValueError(f"{name}: {dtype} expected, got {t.dtype}")
    if t.numel() < n:
        raise ValueError(f"{name}: at least {n} elements expected, got {t.numel()}")
    if device is not None and t.get_device() != device:
        raise ValueError(f"{name}: on device {t.get_device()}, expected {device}")
    return t.data_ptr()


def _rows_ptr(t) -> int:
    """Device pointer of a 2-D tensor whose rows are contiguous (any row pitch)."""
    if not t.is_cuda:
        raise ValueError("device tensor expected")
    if t.dim() != 2 or (t.numel() > 0 and t.stride(1) != 1):
        raise ValueError("2-D tensor with contiguous rows expected")
    return t.data_ptr()


def _row_pitch(t) -> int:
    """Elements between rows (an empty tensor has no rows to step over: its width)."""
    return t.stride(0) if t.numel() > 0 else t.shape[1]


class AttentionCall:
    """``dard_step_attention`` with everything but q, k, v and o marshalled once.

    One step's per-sequence metadata and mask inputs (states, c_{t-1}, shadow sources) are
    the same for every layer, so a caller running many layers builds this once per step and
    calls it per layer. The host arrays are copied; the device tensors are referenced and
    must stay alive and unchanged in size while the object is used. Each call checks q, k,
    v and o against the row count the metadata implies (sum of n_orig + shadow_len), sets
    the four pointers and the stream, and calls the library.

    ``rope_theta`` > 0 makes the call apply RoPE (base theta, pairing ``rope_style``) to q
    and k, which then arrive before RoPE; every call then needs ``k_rope``, a tensor shaped
    like k that receives the rotated keys (k itself rotates k in place)."""

    def __init__(self, n_orig, block_start, block_len, shadow_len, state, prev_conf,
                 shadow_src, scale: float = 0.0, status=None, query_start=None,
                 rope_theta: float = 0.0, rope_style: int = DARD_ROPE_INTERLEAVED):
        torch = _torch()
        self._host = [_host_i32(x) for x in (n_orig, block_start, block_len, shadow_len)]
        self._qs = _host_i32(query_start) if query_start is not None else None
        n, b0, bl, sl = self._host
        ns = len(n)
        if any(len(x) != ns for x in self._host[1:]) or (self._qs is not None and
                                                        len(self._qs) != ns):
            raise ValueError("per-sequence arrays differ in length")
        self.rows = int(n.astype(np.int64).sum() + sl.astype(np.int64).sum())
        blk, sh = int(bl.astype(np.int64).sum()), int(sl.astype(np.int64).sum())
        self.device = state.get_device() if state is not None else None
        a = AttnArgs()
        a.num_seqs = ns
        a.n_orig, a.block_start, a.block_len, a.shadow_len = (
            x.ctypes.data_as(_I32P) for x in self._host)
        a.query_start = self._qs.ctypes.data_as(_I32P) if self._qs is not None else None
        a.state = _dev(state, "state", blk, torch.uint8)
        a.prev_conf = _dev(prev_conf, "prev_conf", blk, torch.float32, self.device)
        a.shadow_src = _dev(shadow_src, "shadow_src", sh, torch.int32, self.device)
        a.status = _dev(status, "status", 1, torch.int32, self.device)
        a.scale = scale
        a.rope_theta = rope_theta
        a.rope_style = rope_style
        self.rope = rope_theta != 0.0
        self._keep = (state, prev_conf, shadow_src, status)
        self._args = a
        self._ref = ctypes.byref(a)
        self._fn = lib().dard_step_attention

    def __call__(self, q, k, v, o, stream=None, k_rope=None):
        """Masked attention of one layer; q/o [rows, hq, d], k/v [rows, hkv, d]; with RoPE,
        ``k_rope`` (like k) receives the rotated keys."""
        dev = self._bind(q, k, v, o, k_rope)
        _check(self._fn(self._ref, _stream_handle(stream, dev)), "dard_step_attention")

    def kernel(self, q, k, v, o) -> int:
        """The kernel a call on these tensors launches, without launching it: 1 or 2 (the
        tensor-core kernel with one or two query tiles per CTA), 4 (the CTA-pair kernel),
        3 (fp32 CUDA cores), 0 (no query rows)."""
        self._bind(q, k, v, o, k if self.rope else None)
        out = ctypes.c_int32(-1)
        _check(lib().dard_attention_kernel(self._ref, ctypes.byref(out)), "dard_attention_kernel")
        return int(out.value)

    def plan(self, q, k, v, o) -> dict:
        """The launch plan of a call on these tensors, without launching it: the kernel, its
        CTAs, and the (query tile, key tile) pairs it computes and skips."""
        self._bind(q, k, v, o, k if self.rope else None)
        out = AttnPlan()
        _check(lib().dard_attention_plan(self._ref, ctypes.byref(out)), "dard_attention_plan")
        return {"kernel": int(out.kernel), "ctas": int(out.ctas),
                "tile_pairs": int(out.tile_pairs),
                "tile_pairs_skipped": int(out.tile_pairs_skipped)}

    def _bind(self, q, k, v, o, k_rope=None) -> int:
        """Checks q, k, v, o (and k_rope) against the metadata and sets their pointers;
        returns the device index."""
        if not (q.is_cuda and k.is_cuda and v.is_cuda and o.is_cuda):
            raise ValueError("q, k, v and o must be device tensors")
        if not (q.is_contiguous() and k.is_contiguous() and v.is_contiguous()
                and o.is_contiguous()):
            raise ValueError("q, k, v and o must be contiguous")
        qs, ks = q.shape, k.shape
        if (len(qs) != 3 or len(ks) != 3 or o.shape != qs or v.shape != ks or ks[2] != qs[2]
                or qs[0] < self.rows or ks[0] < self.rows):
            raise ValueError(f"q/o [>={self.rows}, hq, d] and k/v [>={self.rows}, hkv, d] "
                             f"expected, got {tuple(qs)}, {tuple(ks)}, {tuple(v.shape)}, "
                             f"{tuple(o.shape)}")
        dt = q.dtype
        if k.dtype != dt or v.dtype != dt or o.dtype != dt:
            raise ValueError("q, k, v and o need one dtype")
        dev = q.get_device()
        if (k.get_device() != dev or v.get_device() != dev or o.get_device() != dev
                or (self.device is not None and dev != self.device)):
            raise ValueError("q, k, v, o and the mask inputs need one device")
        if k_rope is not None and (not k_rope.is_cuda or k_rope.shape != ks or
                                   k_rope.dtype != dt or k_rope.get_device() != dev or
                                   not k_rope.is_contiguous()):
            raise ValueError("k_rope must be a contiguous device tensor like k")
        a = self._args
        a.q, a.k, a.v, a.o = q.data_ptr(), k.data_ptr(), v.data_ptr(), o.data_ptr()
        a.k_rope = k_rope.data_ptr() if k_rope is not None else None
        a.dtype = _dtype_code(q)
        a.hq, a.hkv, a.head_dim = qs[1], ks[1], qs[2]
        return dev


def dard_step_attention(q, k, v, o, n_orig, block_start, block_len, shadow_len, state,
                        prev_conf, shadow_src, scale: float = 0.0, status=None, stream=None,
                        query_start=None, rope_theta: float = 0.0,
                        rope_style: int = DARD_ROPE_INTERLEAVED, k_rope=None):
    """Masked attention of one layer; q/o [rows, hq, d], k/v [rows, hkv, d] on the device.
    ``query_start`` (per sequence, optional): first query row; earlier rows are keys only.
    ``rope_theta`` > 0: q and k arrive before RoPE, ``k_rope`` receives the rotated keys."""
    AttentionCall(n_orig, block_start, block_len, shadow_len, state, prev_conf, shadow_src,
                  scale=scale, status=status, query_start=query_start, rope_theta=rope_theta,
                  rope_style=rope_style)(q, k, v, o, stream, k_rope=k_rope)


def dard_attention_kernel(q, k, v, o, n_orig, block_start, block_len, shadow_len, state,
                          prev_conf, shadow_src, scale: float = 0.0, query_start=None) -> int:
    """The kernel dard_step_attention would launch for these arguments (see
    ``AttentionCall.kernel``), without launching anything."""
    return AttentionCall(n_orig, block_start, block_len, shadow_len, state, prev_conf,
                         shadow_src, scale=scale, query_start=query_start).kernel(q, k, v, o)


def dard_score_workspace_size(rows: int, vocab: int, num_seqs: int) -> int:
    return int(lib().dard_score_workspace_size(rows, vocab, num_seqs))


class ScoreCall:
    """``dard_score_and_transition`` with everything but the two logits tensors marshalled
    once: the block lengths, thresholds and every state and output buffer. A decode loop
    builds it once per block (or once, with in-place states) and calls it each step on that
    step's logits. The device tensors are referenced and must stay alive and unchanged in
    size while the object is used. ``workspace=None`` selects
    ``dard_score_and_transition_noalloc`` (the library's built-in scratch)."""

    def __init__(self, block_len, state_in, tau_c, tau_u, lam, p0, conf, token, state_out,
                 workspace, w_out=None, counts=None, status=None, cur_token=None, p_cur=None,
                 tokens=None, mask_token: int = 0, entropy=None, margin=None, order_key=None,
                 order_mode: int = ORDER_CONFIDENCE):
        torch = _torch()
        self._bl = _host_i32(block_len)
        ns = len(self._bl)
        self.rows = rows = int(self._bl.astype(np.int64).sum())
        self.device = dev = state_in.get_device() if state_in is not None else None
        f32, i32, u8 = torch.float32, torch.int32, torch.uint8
        a = ScoreArgs()
        a.num_seqs = ns
        a.block_len = self._bl.ctypes.data_as(_I32P)
        a.state_in = _dev(state_in, "state_in", rows, u8)
        a.tau_c, a.tau_u, a.lambda_, a.p0 = tau_c, tau_u, lam, p0
        a.conf = _dev(conf, "conf", rows, f32, dev)
        a.token = _dev(token, "token", rows, i32, dev)
        a.state_out = _dev(state_out, "state_out", rows, u8, dev)
        a.w_out = _dev(w_out, "w_out", rows, f32, dev)
        a.counts = _dev(counts, "counts", 3 * ns, i32, dev)
        a.status = _dev(status, "status", 1, i32, dev)
        a.cur_token = _dev(cur_token, "cur_token", rows, i32, dev)
        a.p_cur = _dev(p_cur, "p_cur", rows, f32, dev)
        a.tokens = _dev(tokens, "tokens", rows, i32, dev)
        a.mask_token = mask_token
        a.entropy = _dev(entropy, "entropy", rows, f32, dev)
        a.margin = _dev(margin, "margin", rows, f32, dev)
        a.order_key = _dev(order_key, "order_key", rows, f32, dev)
        a.order_mode = order_mode
        if workspace is not None:
            a.workspace = _dev(workspace, "workspace", 0, workspace.dtype, dev)
            a.workspace_bytes = workspace.numel() * workspace.element_size()
            self._fn, self._name = lib().dard_score_and_transition, "dard_score_and_transition"
        else:
            self._fn = lib().dard_score_and_transition_noalloc
            self._name = "dard_score_and_transition_noalloc"
        self._keep = (state_in, conf, token, state_out, w_out, counts, status, cur_token,
                      p_cur, tokens, entropy, margin, order_key, workspace)
        self._args = a
        self._ref = ctypes.byref(a)

    def __call__(self, logits_x, logits_s, stream=None):
        """Scores every block row; logits [rows, V] with contiguous rows and one row pitch
        (``stride(0)``, at least V) in both tensors."""
        shp = logits_s.shape
        if logits_x.shape != shp or len(shp) != 2 or shp[0] < self.rows:
            raise ValueError(f"logits_x and logits_s [>={self.rows}, V] of one shape expected, "
                             f"got {tuple(logits_x.shape)} and {tuple(shp)}")
        pitch = _row_pitch(logits_s)
        if _row_pitch(logits_x) != pitch:
            raise ValueError("logits_x and logits_s need the same row pitch")
        if logits_x.dtype != logits_s.dtype:
            raise ValueError("logits_x and logits_s need one dtype")
        a = self._args
        a.logits_x, a.logits_s = _rows_ptr(logits_x), _rows_ptr(logits_s)
        dev = logits_s.get_device()
        if logits_x.get_device() != dev or (self.device is not None and dev != self.device):
            raise ValueError("the logits and the state and output buffers need one device")
        a.dtype = _dtype_code(logits_s)
        a.vocab = shp[1]
        a.row_stride = pitch
        _check(self._fn(self._ref, _stream_handle(stream, dev)), self._name)


def dard_score_and_transition(logits_x, logits_s, block_len, state_in, tau_c, tau_u, lam, p0,
                              conf, token, state_out, workspace, w_out=None, counts=None,
                              status=None, stream=None, cur_token=None, p_cur=None,
                              tokens=None, mask_token: int = 0, entropy=None, margin=None,
                              order_key=None, order_mode: int = ORDER_CONFIDENCE):
    """Scoring and transition of every block row; logits [rows, V] with contiguous rows and
    the same row pitch (``stride(0)``, at least V) in both tensors. Optional end of step:
    ``p_cur`` of ``cur_token``, and ``tokens`` (x^, or ``mask_token`` for rows ending in M);
    ``entropy``, ``margin`` and the next step's ``order_key`` for ``order_mode``."""
    if workspace is None:
        raise ValueError("workspace is required (see dard_score_workspace_size)")
    ScoreCall(block_len, state_in, tau_c, tau_u, lam, p0, conf, token, state_out, workspace,
              w_out=w_out, counts=counts, status=status, cur_token=cur_token, p_cur=p_cur,
              tokens=tokens, mask_token=mask_token, entropy=entropy, margin=margin,
              order_key=order_key, order_mode=order_mode)(logits_x, logits_s, stream)


def dard_score_and_transition_noalloc(logits_x, logits_s, block_len, state_in, tau_c, tau_u,
                                      lam, p0, conf, token, state_out, w_out=None, counts=None,
                                      status=None, stream=None):
    """``dard_score_and_transition`` without a workspace: the library's built-in scratch
    (at most ``SCORE_NOALLOC_MAX_ROWS`` block rows; calls that overlap on one device race)."""
    ScoreCall(block_len, state_in, tau_c, tau_u, lam, p0, conf, token, state_out, None,
              w_out=w_out, counts=counts, status=status)(logits_x, logits_s, stream)


# ------------------------------------------------------------------ experts' MLP (MXFP8)
def mx_scale_shape(shape, layout: int = MX_SCALE_ROWS) -> tuple:
    """Shape of the uint8 scale tensor of a [rows, cols] matrix or a [batch, rows, cols] batch:
    layout ROWS [..., rows, cols / 32 rounded up to 16], layout TILES [..., row tiles, column
    tiles, 512]."""
    *lead, rows, cols = shape
    if cols % MX_BLOCK:
        raise ValueError(f"rows of {cols} elements are no multiple of {MX_BLOCK}")
    if layout == MX_SCALE_ROWS:
        return (*lead, rows, -(-cols // (16 * MX_BLOCK)) * 16)
    return (*lead, -(-rows // 128), -(-cols // 128), 512)


def _is_dtype(t, name: str, dtypes):
    if t.dtype not in dtypes:
        raise ValueError(f"{name}: {' or '.join(str(d) for d in dtypes)} expected, got {t.dtype}")


def _types() -> dict:
    """The accepted dtypes of codes, scales and the other tensors."""
    torch = _torch()
    return {"codes": (torch.float8_e4m3fn, torch.uint8),
            "scales": (torch.uint8, torch.float8_e8m0fnu), "bf16": (torch.bfloat16,),
            "f32": (torch.float32,), "i32": (torch.int32,),
            "float": (torch.bfloat16, torch.float32)}


_TYPES: dict = {}


def _dtypes(kind: str) -> tuple:
    if not _TYPES:
        _TYPES.update(_types())
    return _TYPES[kind]


def _rows2(t, name: str, shape: tuple, dtypes: tuple, device: int) -> tuple[int, int]:
    """(pointer, row stride) of a device tensor of this 2-D shape with contiguous rows. (One
    pass of cheap comparisons; what is wrong is looked for only when one fails.)"""
    if t.dtype in dtypes and t.get_device() == device >= 0 and t.shape == shape:
        s0, s1 = t.stride()
        if s1 == 1 and s0 >= shape[1]:
            return t.data_ptr(), s0
    if not t.is_cuda:
        raise ValueError(f"{name}: device tensor expected")
    if t.get_device() != device:
        raise ValueError(f"{name}: on device {t.get_device()}, expected {device}")
    _is_dtype(t, name, dtypes)
    if tuple(t.shape) != tuple(shape):
        raise ValueError(f"{name}: {list(shape)} expected, got {tuple(t.shape)}")
    rows, cols = shape
    if cols > 1 and rows > 0 and t.stride(1) != 1:
        raise ValueError(f"{name}: contiguous rows expected")
    if rows > 1 and t.stride(0) < cols:
        raise ValueError(f"{name}: rows overlap (row stride {t.stride(0)})")
    return t.data_ptr(), max(t.stride(0), cols)  # a stride that no step uses may be anything


def _scale_rows(t, name: str, rows: int, cols: int, device: int) -> tuple[int, int]:
    """(pointer, pitch) of a scale tensor in layout ROWS for [rows, cols] elements."""
    shape = t.shape
    if len(shape) != 2 or shape[1] * MX_BLOCK < cols:
        raise ValueError(f"{name}: {list(mx_scale_shape((rows, cols)))} expected, got {tuple(shape)}")
    return _rows2(t, name, (rows, shape[1]), _dtypes("scales"), device)


def _packed_fn(name: str):
    """The library's function ``name`` for arguments packed into a bytes object: one per call, so
    that threads may share a prepared call (the library runs without the interpreter lock)."""
    f = lib()[name]  # (an object of its own, with its own argument types)
    f.restype, f.argtypes = ctypes.c_int, [ctypes.c_void_p, ctypes.c_void_p]
    return f


class NormCall:
    """``dard_residual_norm`` with the weight and epsilon of one norm marshalled once.

    Call it with ``x`` [rows, dim] and any of the outputs: ``residual`` receives x + ``delta``
    (x itself without delta) and may be x or delta; ``y`` the norm in x's dtype; ``y8`` (e4m3 or
    uint8) and ``y8_scale`` (layout ROWS, see ``mx_scale_shape``) the norm in MXFP8. Threads may
    share this and the MLP's other calls (workspaces are a stream's: calls that overlap on the GPU
    need their own)."""

    layout = struct.Struct("=7Qii7qf4x")  # dard_norm_args

    def __init__(self, dim: int, dtype, weight=None, eps: float = 1e-6):
        if dtype not in _dtypes("float"):
            raise ValueError(f"unsupported dtype {dtype}")
        self.dim, self._dt = dim, (dtype,)
        self._codes = _dtypes("codes")
        if weight is not None and weight.numel() != dim:
            raise ValueError(f"weight: {dim} elements expected, got {weight.numel()}")
        self.device = None if weight is None else weight.get_device()
        self._weight_ptr = _dev(weight, "weight", dim, dtype) or 0
        self._weight = weight
        self._eps = eps
        self._code = DARD_BF16 if dtype == _torch().bfloat16 else DARD_F32
        self._fn = _packed_fn("dard_residual_norm")

    def __call__(self, x, delta=None, residual=None, y=None, y8=None, y8_scale=None, stream=None):
        dim, dt, dev = self.dim, self._dt, x.get_device()
        if self.device is not None and dev != self.device:
            raise ValueError(f"x: on device {dev}, the weight on {self.device}")
        rows = x.shape[0]
        shape = (rows, dim)
        xp, xs = _rows2(x, "x", shape, dt, dev)
        dp, ds = _rows2(delta, "delta", shape, dt, dev) if delta is not None else (0, 0)
        rp, rs = _rows2(residual, "residual", shape, dt, dev) if residual is not None else (0, 0)
        yp, ys = _rows2(y, "y", shape, dt, dev) if y is not None else (0, 0)
        qp = qs = sp = ss = 0
        if y8 is not None:
            if y8_scale is None:
                raise ValueError("y8 needs y8_scale")
            qp, qs = _rows2(y8, "y8", shape, self._codes, dev)
            sp, ss = _scale_rows(y8_scale, "y8_scale", rows, dim, dev)
        args = self.layout.pack(xp, dp, self._weight_ptr, rp, yp, qp, sp, self._code, dim, rows, xs,
                                ds, rs, ys, qs, ss, self._eps)
        _check(self._fn(args, _stream_handle(stream, dev)), "dard_residual_norm")


def dard_residual_norm(x, delta=None, weight=None, eps: float = 1e-6, residual=None, y=None,
                       y8=None, y8_scale=None, stream=None):
    """Residual addition and root-mean-square norm of the rows of x, see ``NormCall``."""
    NormCall(x.shape[-1], x.dtype, weight, eps)(x, delta, residual, y, y8, y8_scale, stream)


_MX_LAYOUT = struct.Struct("=3Qiiiiqqqq")  # dard_mx_args


def _flat(t, name: str, dtypes: tuple, device: int, least: int = 0) -> int:
    """Pointer of a contiguous device tensor of at least ``least`` elements."""
    if t.dtype not in dtypes or not t.get_device() == device >= 0 or not t.is_contiguous():
        _is_dtype(t, name, dtypes)
        raise ValueError(f"{name}: contiguous tensor on device {device} expected")
    if t.numel() < least:
        raise ValueError(f"{name}: at least {least} elements expected, got {t.numel()}")
    return t.data_ptr()


def dard_mx_quantize(x, codes, scales, layout: int = MX_SCALE_ROWS, stream=None):
    """MXFP8 rounding of x [rows, cols] or [batch, rows, cols] (contiguous rows, any row and batch
    stride) into contiguous ``codes`` of x's shape and ``scales`` of ``mx_scale_shape``."""
    if not x.is_cuda:
        raise ValueError("x: device tensor expected")
    dev, shp, strides = x.get_device(), x.shape, x.stride()
    if len(shp) not in (2, 3) or (strides[-1] != 1 and shp[-1] > 1):
        raise ValueError("x: [rows, cols] or [batch, rows, cols] with contiguous rows expected")
    if codes.shape != shp:
        raise ValueError(f"codes: {tuple(shp)} expected, got {tuple(codes.shape)}")
    by_rows = layout == MX_SCALE_ROWS
    if not by_rows and layout != MX_SCALE_TILES:
        raise ValueError(f"layout {layout} is neither MX_SCALE_ROWS nor MX_SCALE_TILES")
    rows, cols = shp[-2], shp[-1]
    batch = shp[0] if len(shp) == 3 else 1
    got = scales.shape
    if (got[:-1] != shp[:-1] or got[-1] * MX_BLOCK < cols) if by_rows else \
            got != mx_scale_shape(shp, layout):
        raise ValueError(f"scales: {mx_scale_shape(shp, layout)} expected, got {tuple(got)}")
    a = MxArgs()
    # (a stride that no step uses may be anything)
    _MX_LAYOUT.pack_into(
        a, 0, x.data_ptr(), _flat(codes, "codes", _dtypes("codes"), dev),
        _flat(scales, "scales", _dtypes("scales"), dev), _dtype_code(x), layout, batch, cols, rows,
        strides[-2] if rows > 1 else cols, strides[0] if batch > 1 else 0, got[-1] if by_rows else 0)
    _check(lib().dard_mx_quantize(ctypes.byref(a), _stream_handle(stream, dev)),
           "dard_mx_quantize")


def dard_route_workspace_size(tokens: int, experts: int, top_k: int) -> int:
    return int(lib().dard_route_workspace_size(tokens, experts, top_k))


class RouteCall:
    """``dard_route`` with a router's settings and its bias marshalled once.

    With ``top_groups`` < ``groups`` a group's rank is the sum of its two largest choices.
    Call it with logits [tokens, experts] (bf16 or fp32, contiguous rows), ``ids`` and
    ``weights`` [tokens, top_k], and, for the plan that ``ExpertsCall`` reads, ``offsets``
    [experts + 1] and ``rows`` [tokens * top_k]. The workspace holds
    ``dard_route_workspace_size`` bytes for the most tokens of a call with a plan, which are
    enough for fewer tokens too."""

    layout = struct.Struct("=QqQ8if4x6QQ")  # dard_route_args

    def __init__(self, experts: int, top_k: int, scoring: int = ROUTE_SOFTMAX, bias=None,
                 groups: int = 1, top_groups: int = 1, renormalise: bool = True,
                 scale: float = 1.0, workspace=None, status=None):
        torch = _torch()
        self.experts, self.top_k = experts, top_k
        self.device = next((t.get_device() for t in (bias, workspace, status) if t is not None), None)
        self._bias = _dev(bias, "bias", experts, torch.float32, self.device) or 0
        self._scoring = scoring
        self._settings = (experts, top_k, groups, top_groups, 1 if renormalise else 0, scale)
        status_ptr = _dev(status, "status", 1, torch.int32, self.device) or 0
        self._scratch = (status_ptr, 0, 0)
        if workspace is not None:
            self._scratch = (status_ptr,
                             _dev(workspace, "workspace", 0, workspace.dtype, self.device),
                             workspace.numel() * workspace.element_size())
        self._keep = (bias, workspace, status)
        self._fn = _packed_fn("dard_route")

    def __call__(self, logits, ids, weights, offsets=None, rows=None, stream=None):
        k, tokens, dev = self.top_k, logits.shape[0], logits.get_device()
        if self.device is not None and dev != self.device:
            raise ValueError(f"logits: on device {dev}, expected {self.device}")
        lp, ls = _rows2(logits, "logits", (tokens, self.experts), _dtypes("float"), dev)
        if ids.shape != (tokens, k) or weights.shape != (tokens, k):
            raise ValueError(f"ids and weights: [{tokens}, {k}] expected, got {tuple(ids.shape)}, "
                             f"{tuple(weights.shape)}")
        i32 = _dtypes("i32")
        ip, wp = _flat(ids, "ids", i32, dev), _flat(weights, "weights", _dtypes("f32"), dev)
        if (offsets is None) != (rows is None):
            raise ValueError("offsets and rows come together")
        op = rp = 0
        if offsets is not None:
            op = _flat(offsets, "offsets", i32, dev, self.experts + 1)
            rp = _flat(rows, "rows", i32, dev, tokens * k)
        args = self.layout.pack(lp, ls, self._bias, _dtype_code(logits), self._scoring, tokens,
                                *self._settings, ip, wp, op, rp, *self._scratch)
        _check(self._fn(args, _stream_handle(stream, dev)), "dard_route")


def dard_route(logits, ids, weights, top_k: int, scoring: int = ROUTE_SOFTMAX, bias=None,
               groups: int = 1, top_groups: int = 1, renormalise: bool = True, scale: float = 1.0,
               offsets=None, rows=None, workspace=None, status=None, stream=None):
    """Experts and weights of each row of logits, and the plan, see ``RouteCall``."""
    RouteCall(logits.shape[-1], top_k, scoring, bias, groups, top_groups, renormalise, scale,
              workspace, status)(logits, ids, weights, offsets, rows, stream)


def dard_experts_workspace_size(tokens: int, experts: int, top_k: int, dim: int,
                                hidden: int) -> int:
    return int(lib().dard_experts_workspace_size(tokens, experts, top_k, dim, hidden))


class ExpertsCall:
    """``dard_experts`` with one layer's weights and the workspace marshalled once.

    w1 and w3 are [experts, hidden, dim], w2 [experts, dim, hidden], contiguous: bf16 (scales
    None), or e4m3 / uint8 codes with uint8 / e8m0 scales in layout TILES (``dard_mx_quantize``).
    Call it with x [tokens, dim] (x_scale in layout ROWS for MXFP8), the outputs of a
    ``RouteCall`` and y [tokens, dim] in bf16 or fp32. The workspace holds
    ``dard_experts_workspace_size`` bytes for the most tokens of a call, which are enough for
    fewer tokens too."""

    layout = struct.Struct("=13Q3q7i4x3Q")  # dard_experts_args

    def __init__(self, w1, w1_scale, w3, w3_scale, w2, w2_scale, workspace, status=None):
        torch = _torch()
        if w1.dim() != 3 or w3.shape != w1.shape or tuple(w2.shape) != (
                w1.shape[0], w1.shape[2], w1.shape[1]):
            raise ValueError("w1 and w3 [experts, hidden, dim] and w2 [experts, dim, hidden] expected, "
                             f"got {tuple(w1.shape)}, {tuple(w3.shape)}, {tuple(w2.shape)}")
        self.experts, self.hidden, self.dim = w1.shape
        self.mx = w1.dtype != torch.bfloat16
        self._bf16 = torch.bfloat16
        self.device = dev = w1.get_device()
        codes, scales = [], []  # w1, w3, w2
        for name, w, s in (("w1", w1, w1_scale), ("w3", w3, w3_scale), ("w2", w2, w2_scale)):
            _is_dtype(w, name, _dtypes("codes" if self.mx else "bf16"))
            codes.append(_dev(w, name, w.numel(), w.dtype, dev))
            if not self.mx:
                if s is not None:
                    raise ValueError(f"{name}_scale: bf16 weights have no scales")
                continue
            if s is None:
                raise ValueError(f"{name}_scale: needed with 8-bit weights")
            want = mx_scale_shape(w.shape, MX_SCALE_TILES)
            _is_dtype(s, name + "_scale", _dtypes("scales"))
            if tuple(s.shape) != want:
                raise ValueError(f"{name}_scale: {want} expected, got {tuple(s.shape)}")
            scales.append(_dev(s, name + "_scale", s.numel(), s.dtype, dev))
        self._weights = (*codes, *(scales or (0, 0, 0)))
        self._code = DARD_MXFP8 if self.mx else DARD_BF16
        if workspace is None:
            raise ValueError("workspace is required (see dard_experts_workspace_size)")
        self._scratch = (_dev(workspace, "workspace", 0, workspace.dtype, dev),
                         workspace.numel() * workspace.element_size(),
                         _dev(status, "status", 1, torch.int32, dev) or 0)
        self._keep = (w1, w1_scale, w3, w3_scale, w2, w2_scale, workspace, status)
        self._fn = _packed_fn("dard_experts")

    def __call__(self, x, x_scale, ids, weights, offsets, rows, y, stream=None):
        dev, dim = self.device, self.dim
        tokens, k = ids.shape
        shape = (tokens, dim)
        xp, xs = _rows2(x, "x", shape, _dtypes("codes" if self.mx else "bf16"), dev)
        sp = ss = 0
        if self.mx:
            if x_scale is None:
                raise ValueError("x_scale: needed with 8-bit weights")
            sp, ss = _scale_rows(x_scale, "x_scale", tokens, dim, dev)
        yp, ys = _rows2(y, "y", shape, _dtypes("float"), dev)
        if weights.shape != ids.shape:
            raise ValueError(f"weights: {tuple(ids.shape)} expected, got {tuple(weights.shape)}")
        i32, f32 = _dtypes("i32"), _dtypes("f32")
        ip, wp = _flat(ids, "ids", i32, dev), _flat(weights, "weights", f32, dev)
        op = _flat(offsets, "offsets", i32, dev, self.experts + 1)
        rp = _flat(rows, "rows", i32, dev, tokens * k)
        args = self.layout.pack(
            xp, sp, *self._weights, ip, wp, op, rp, yp, xs, ss, ys, self._code,
            DARD_BF16 if y.dtype == self._bf16 else DARD_F32, tokens, self.experts, k, dim,
            self.hidden, *self._scratch)
        _check(self._fn(args, _stream_handle(stream, dev)), "dard_experts")


def dard_experts(x, x_scale, w1, w1_scale, w3, w3_scale, w2, w2_scale, ids, weights, offsets,
                 rows, y, workspace, status=None, stream=None):
    """The experts' products of every token, weighted and added, see ``ExpertsCall``."""
    ExpertsCall(w1, w1_scale, w3, w3_scale, w2, w2_scale, workspace, status)(
        x, x_scale, ids, weights, offsets, rows, y, stream)
