"""The MLP half of a layer with experts: residual addition, norm, routing and the experts.

``ExpertMLP`` owns one layer's weights in the form that the kernels read (MXFP8 codes with
scales in tiles, rounded once from the given weights, or bf16) and the buffers of a call; its
call runs ``dard_residual_norm``, the router's product (a plain library GEMM), ``dard_route`` and
``dard_experts`` on the current stream, with no host round trip between them. A dense MLP is the
case of one expert.
"""
from __future__ import annotations

import torch

from . import binding as B


def mx_weights(w: torch.Tensor) -> tuple[torch.Tensor, torch.Tensor]:
    """(e4m3 codes, scales in tiles) of weights [experts, rows, cols]."""
    codes = torch.empty(w.shape, dtype=torch.float8_e4m3fn, device=w.device)
    scales = torch.empty(B.mx_scale_shape(w.shape, B.MX_SCALE_TILES), dtype=torch.uint8,
                         device=w.device)
    B.dard_mx_quantize(w, codes, scales, B.MX_SCALE_TILES)
    return codes, scales


class ExpertMLP:
    """One layer's norm, router and experts.

    w1, w3 [experts, hidden, dim] (gate and value), w2 [experts, dim, hidden] and router
    [dim, experts] in the model's dtype (bf16 or fp32). ``mx``: weights and activations of the
    products in MXFP8; without it they stay bf16 (a bf16 model's only). ``route`` holds further
    arguments of ``RouteCall`` (scoring, bias, groups, ...). ``status`` (int32, one word; the layer's
    own one if none is given) collects the kernels' status bits: the caller reads it, for after
    ``STATUS_TIMEOUT`` outputs are unwritten, and ``STATUS_INVALID_ROW`` marks rows whose router
    logits were NaN or +inf, which get no expert. ``workspaces`` (a dict) may be shared by
    the layers of a model, which run one after another.

    The buffers of a call are kept, one set for each stream and each power of two of tokens from 32
    on: whatever token counts come, there are few sets, each of about half the size of the next;
    calls on different streams share none, and a set's addresses stay what a captured graph holds. One thread at a
    time calls the layers that share a dict on one stream."""

    _MAX_PREPARED = 256  # token counts (and streams) whose views and calls are kept

    def __init__(self, w1, w3, w2, router, top_k: int, norm_weight=None, eps: float = 1e-6,
                 mx: bool = True, route: dict | None = None, status=None,
                 workspaces: dict | None = None):
        if not router.is_cuda:
            raise ValueError("router: device tensor expected")
        self.experts, self.hidden, self.dim = w1.shape
        self.top_k, self.dtype, self.mx = top_k, router.dtype, mx
        if not mx and router.dtype != torch.bfloat16:
            raise ValueError("products without MXFP8 need bf16 weights")
        self.router = router
        weights = (w1, w3, w2)
        if mx:
            self.weights = [t for w in weights for t in mx_weights(w)]
        else:
            self.weights = [t for w in weights for t in (w, None)]
        self.status = status if status is not None else torch.zeros(
            1, dtype=torch.int32, device=router.device)
        self.norm = B.NormCall(self.dim, router.dtype, norm_weight, eps)
        self._route = dict(route or {})
        self._shared = {} if workspaces is None else workspaces
        # by stream and token count: views of the buffers, routing, experts
        self._calls: dict[tuple, tuple] = {}

    def _buffers(self, stream: int, tokens: int) -> dict:
        """Workspaces and intermediate tensors for up to ``tokens`` rows on a stream."""
        dev, dim, k = self.router.device, self.dim, self.top_k
        key = (dev, stream, tokens, self.experts, k, dim, self.hidden, self.mx, self.dtype)
        b = self._shared.get(key)
        if b is None:
            def empty(*shape, dtype):
                return torch.empty(shape, dtype=dtype, device=dev)

            need_r = B.dard_route_workspace_size(tokens, self.experts, k)
            need_e = B.dard_experts_workspace_size(tokens, self.experts, k, dim, self.hidden)
            b = dict(route_ws=empty(max(need_r, 16), dtype=torch.uint8),
                     experts_ws=empty(max(need_e, 16), dtype=torch.uint8),
                     y=empty(tokens, dim, dtype=self.dtype),
                     logits=empty(tokens, self.experts, dtype=self.dtype),
                     ids=empty(tokens, k, dtype=torch.int32),
                     weights=empty(tokens, k, dtype=torch.float32),
                     offsets=empty(self.experts + 1, dtype=torch.int32),
                     rows=empty(tokens * k, dtype=torch.int32))
            if self.mx:
                b["y8"] = empty(tokens, dim, dtype=torch.float8_e4m3fn)
                b["y8_scale"] = empty(*B.mx_scale_shape((tokens, dim)), dtype=torch.uint8)
            self._shared[key] = b
        return b

    def _prepared(self, tokens: int) -> tuple:
        """(buffers, RouteCall, ExpertsCall) for ``tokens`` rows on the current stream, marshalled
        once."""
        stream = B._raw_stream(self.router.get_device())
        c = self._calls.get((stream, tokens))
        if c is None:
            # the next power of two from 32 on (an expert's rows take whole tiles, so that sets of
            # fewer are hardly smaller), as far as the products take so many tokens
            most = min(1 << max(tokens - 1, 31).bit_length(), B.EXPERTS_MAX_PAIRS // self.top_k)
            b = dict(self._buffers(stream, max(most, tokens)))
            for name in ("y", "logits", "ids", "weights", "y8", "y8_scale"):
                if name in b:
                    b[name] = b[name][:tokens]
            b["rows"] = b["rows"][:tokens * self.top_k]
            c = (b, B.RouteCall(self.experts, self.top_k, workspace=b["route_ws"],
                                status=self.status, **self._route),
                 B.ExpertsCall(*self.weights, workspace=b["experts_ws"], status=self.status))
            if len(self._calls) >= self._MAX_PREPARED:
                self._calls.clear()
            self._calls[stream, tokens] = c
        return c

    def __call__(self, h: torch.Tensor, delta: torch.Tensor | None = None,
                 out: torch.Tensor | None = None) -> torch.Tensor:
        """The MLP's output for residual rows h [tokens, dim], with ``delta`` (the attention's
        output) added to h in place first. The caller adds the result to h (its next norm can)."""
        b, route, experts = self._prepared(h.shape[0])
        out = torch.empty_like(b["y"]) if out is None else out
        self.norm(h, delta, residual=h if delta is not None else None, y=b["y"], y8=b.get("y8"),
                  y8_scale=b.get("y8_scale"))
        torch.mm(b["y"], self.router, out=b["logits"])
        route(b["logits"], b["ids"], b["weights"], b["offsets"], b["rows"])
        x, scale = (b["y8"], b["y8_scale"]) if self.mx else (b["y"], None)
        experts(x, scale, b["ids"], b["weights"], b["offsets"], b["rows"], out)
        return out
