"""CPU oracle of decoding behind a shared prefix, in float64 NumPy straight from the definitions:
attention over the prefix and each sequence's own rows, the weight that each key of the prefix has
received, and the keys to keep. It shares no code with the CUDA path; the mask over a sequence's own
rows is ``dard_oracle.attention_mask``.

With each result comes what its rounding errors scale with, so that a test can state its tolerance
elementwise: ``mass`` = sum_j p_j |v_j| for an output, ``dot`` = the largest sum_i |q_i k_i| times the
scale behind a score of the row or key.
"""
from __future__ import annotations

import math

import numpy as np

from oracle import dard_oracle as D


def prefix_attention(q, k, v, pk, pv, layouts, query_start=None, scale=None):
    """(o, lse, mass, dot) of every row; rows that are no queries, and shadow rows that are no valid
    ones, are NaN. q [R, Hq, d], k and v [R, Hkv, d], pk and pv [P, Hkv, d]."""
    rows, hq, d = q.shape
    hkv = k.shape[1]
    scale = 1.0 / math.sqrt(d) if scale is None else scale
    q, k, v, pk, pv = (np.asarray(x, np.float64) for x in (q, k, v, pk, pv))
    o = np.full((rows, hq, d), np.nan)
    lse = np.full((rows, hq), np.nan)
    mass, dot = np.full_like(o, np.nan), np.full_like(lse, np.nan)
    base = 0
    for i, lay in enumerate(layouts):
        first = 0 if query_start is None else int(query_start[i])
        at = np.arange(first, lay.rows)
        mask = D.attention_mask(lay, at)
        see = np.concatenate([np.ones((len(at), len(pk)), bool), mask], 1)
        for h in range(hq):
            g = h // (hq // hkv)
            kk = np.concatenate([pk[:, g], k[base:base + lay.rows, g]])
            vv = np.concatenate([pv[:, g], v[base:base + lay.rows, g]])
            qq = q[base + at, h]
            with np.errstate(invalid="ignore", over="ignore"):
                z = np.where(see, qq @ np.where(np.isfinite(kk), kk, 0.0).T * scale, -np.inf)
                bad = ~np.isfinite(kk).all(1)  # keys with a NaN or an infinity, one by one
                for j in np.nonzero(bad)[0]:
                    z[:, j] = np.where(see[:, j], (qq * kk[j]).sum(1) * scale, -np.inf)
                top = z.max(1, keepdims=True)
                p = np.exp(z - top)
                total = p.sum(1, keepdims=True)
                p = p / total
                fine = np.where(np.isfinite(vv), vv, 0.0)
                out = p @ fine
                for j in np.nonzero(~np.isfinite(vv).all(1))[0]:  # only where the key is seen
                    out += np.where(see[:, j, None] & ~np.isfinite(vv[j]), vv[j], 0.0)
            o[base + at, h] = out
            lse[base + at, h] = (top + np.log(total))[:, 0]
            mass[base + at, h] = p @ np.abs(fine)
            dot[base + at, h] = np.where(see, np.abs(qq) @ np.abs(np.where(np.isfinite(kk), kk, 0)).T,
                                         0).max(1) * scale
        base += lay.rows
    return o, lse, mass, dot


def prefix_weights(q, lse, pk, weights_in=None, decay=1.0, scale=None):
    """(weights, sums without the earlier ones, dot) [Hkv, P]; rows with lse = +inf add nothing."""
    rows, hq, d = q.shape
    hkv = pk.shape[1]
    scale = 1.0 / math.sqrt(d) if scale is None else scale
    q, pk, lse = (np.asarray(x, np.float64) for x in (q, pk, lse))
    new, dot = np.zeros((hkv, len(pk))), np.zeros((hkv, len(pk)))
    for h in range(hq):
        g = h // (hq // hkv)
        use = lse[:, h] != np.inf
        qq = q[use, h]
        if len(qq):
            new[g] += np.exp(qq @ pk[:, g].T * scale - lse[use, h, None]).sum(0)
            dot[g] = np.maximum(dot[g], (np.abs(qq) @ np.abs(pk[:, g]).T).max(0) * scale)
    total = new if weights_in is None else new + decay * np.asarray(weights_in, np.float64)
    return total, new, dot


def prefix_evict(weights, keep, keep_first=0, keep_last=0):
    """kept [Hkv, keep]: one key after the other, the largest that is left, the lowest index first."""
    out = []
    for w in np.asarray(weights, np.float64):
        n = len(w)
        ends = set(range(keep_first)) | set(range(n - keep_last, n))
        middle = [j for j in range(n) if j not in ends]
        rank = sorted(middle, key=lambda j: (np.inf if np.isnan(w[j]) else -w[j], np.isnan(w[j]), j))
        out.append(sorted(ends | set(rank[:keep - keep_first - keep_last])))
    return np.array(out, np.int32).reshape(len(weights), keep)
