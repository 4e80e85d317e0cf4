"""A prefix that a batch shares, cached: its keys and values by layer, the attention weight each key
has received, and their eviction. Wraps ``PrefixAttentionCall``, ``PrefixWeightsCall`` and
``PrefixEvictCall`` (binding.py) with a model's buffers.

One cache serves every sequence that follows the prefix. Its keys carry their positions (RoPE
applied), so that an eviction, after which the heads hold different positions, changes nothing for
the calls that follow."""
from __future__ import annotations

import torch

from . import binding as B


class PrefixCache:
    """Keys and values of a prefix, ``layers`` times [capacity, hkv, head_dim].

    ``store`` fills a layer (the same number of rows in each), ``attention`` prepares a step's calls,
    ``attend`` runs a layer's attention, ``accumulate`` adds the weights of its queries to the layer's,
    and ``evict`` keeps the ``keep`` keys of each head with the largest weights. ``status``: optional
    int32 word that the calls report in. Every prepared attention and every ``accumulate`` has a
    workspace of its own, so that they may overlap, as may graphs that hold them; what they read and
    write of the cache itself is the caller's to order. ``store`` and ``evict`` change lengths and,
    the latter, buffers: a graph captured before one of them holds the cache as it was then."""

    def __init__(self, layers: int, hq: int, hkv: int, head_dim: int, capacity: int,
                 dtype=torch.bfloat16, device="cuda", status=None):
        if layers < 1 or capacity < 1 or hkv < 1 or hq % hkv:
            raise ValueError(f"layers {layers}, capacity {capacity}, heads {hq} / {hkv}")
        self.device = torch.device(device)
        if self.device.type != "cuda":
            raise ValueError("a CUDA device is needed")
        if self.device.index is None:  # (the current device may be another one at a later call)
            self.device = torch.device("cuda", torch.cuda.current_device())
        self.hq, self.hkv, self.head_dim, self.capacity, self.dtype = hq, hkv, head_dim, capacity, dtype
        self.status = status
        # a layer more than the model has: an eviction writes into the spare one, which then takes
        # the evicted layer's place
        self._kv = [torch.empty(2, capacity, hkv, head_dim, dtype=dtype, device=self.device)
                    for _ in range(layers + 1)]
        self._weights = [torch.zeros(hkv, capacity, device=self.device) for _ in range(layers + 1)]
        self._length = [0] * layers
        self._layers = layers
        self.start = 0  # positions that the prefix takes: rows behind it start there
        self._kept = torch.empty(hkv * capacity, dtype=torch.int32, device=self.device)

    @property
    def layers(self) -> int:
        return self._layers

    def length(self, layer: int = 0) -> int:
        """Keys that the layer holds."""
        return self._length[layer]

    def keys(self, layer: int):
        return self._kv[layer][0, :self._length[layer]]

    def values(self, layer: int):
        return self._kv[layer][1, :self._length[layer]]

    def weights(self, layer: int):
        """[hkv, length] weights that the layer's keys have received since they were stored."""
        n = self._length[layer]
        return self._weights[layer].view(-1)[:self.hkv * n].view(self.hkv, n)

    def store(self, layer: int, k, v):
        """The layer's keys (positions applied) and values [rows, hkv, head_dim]; weights start at 0."""
        n = k.shape[0]
        want = (n, self.hkv, self.head_dim)
        if tuple(k.shape) != want or tuple(v.shape) != want or n > self.capacity:
            raise ValueError(f"k and v: [<={self.capacity}, {self.hkv}, {self.head_dim}] expected, got "
                             f"{tuple(k.shape)}, {tuple(v.shape)}")
        self._length[layer] = self.start = n
        self.keys(layer).copy_(k)
        self.values(layer).copy_(v)
        self.weights(layer).zero_()

    def _scratch(self, need: int):
        return torch.empty(need, dtype=torch.uint8, device=self.device) if need else None

    def attention(self, n_orig, block_start, block_len, shadow_len, state, prev_conf, shadow_src,
                  scale: float = 0.0, query_start=None) -> B.PrefixAttentionCall:
        """One step's prepared attention, for ``attend``: see ``PrefixAttentionCall``. (Calls of it share
        its workspace: prepare one for each of those that overlap on the GPU. A graph that captured it
        needs it kept, like every tensor that it was given.)"""
        rows = sum(int(x) for x in n_orig) + sum(int(x) for x in shadow_len)
        need = B.dard_prefix_attention_workspace_size(rows, self.hq, self.hkv, self.head_dim, self.capacity)
        call = B.PrefixAttentionCall(n_orig, block_start, block_len, shadow_len, state, prev_conf,
                                     shadow_src, scale, self.status, query_start, scratch := self._scratch(need))
        call.scratch, call.prepared_on = scratch, B._raw_stream(self.device.index)
        return call

    def attend(self, call: B.PrefixAttentionCall, layer: int, q, k, v, o, lse=None):
        """A layer's attention over the cache and the sequences' own rows."""
        call(q, k, v, o, self.keys(layer), self.values(layer), lse=lse)
        # the workspace belongs to the stream of the preparation: on another one it must outlive the launch,
        # though the call may be dropped right away
        scratch = getattr(call, "scratch", None)  # (a call that was made otherwise has its maker's)
        if scratch is not None and B._raw_stream(self.device.index) != call.prepared_on:
            scratch.record_stream(torch.cuda.current_stream(self.device))

    def accumulate(self, layer: int, q, lse, scale: float = 0.0, decay: float = 1.0):
        """Adds the weights that q's rows spent on the layer's keys to ``decay`` times the earlier ones
        (lse as ``attend`` wrote it; +inf: the row does not count)."""
        if self._length[layer] == 0:
            return
        need = B.dard_prefix_weights_workspace_size(q.shape[0], self.hq, self.hkv, self.head_dim,
                                                    self.capacity)
        w = self.weights(layer)
        B.dard_prefix_weights(q, lse, self.keys(layer), w, weights_in=w, scale=scale, decay=decay,
                              workspace=self._scratch(need), status=self.status)

    def evict(self, keep: int, keep_first: int = 0, keep_last: int = 0):
        """Every layer down to ``keep`` keys per head: the first and last few, and of the others those
        with the largest weights. Layers that hold no more than ``keep`` stay as they are."""
        if keep_first < 0 or keep_last < 0 or keep_first + keep_last > keep:
            raise ValueError(f"keep {keep} with {keep_first} first and {keep_last} last keys")
        call = B.PrefixEvictCall(keep_first, keep_last)
        spare = self._layers
        for layer in range(self._layers):
            if self._length[layer] <= keep:
                continue
            out, w_out = self._kv[spare], self._weights[spare].view(-1)[:self.hkv * keep].view(self.hkv, keep)
            call(self.weights(layer), self.keys(layer), self.values(layer),
                 self._kept[:self.hkv * keep].view(self.hkv, keep), out[0, :keep], out[1, :keep], w_out)
            for buf in (self._kv, self._weights):
                buf[layer], buf[spare] = buf[spare], buf[layer]
            self._length[layer] = keep
