"""CPU oracle of the experts' MLP: MXFP8 rounding, residual + norm, routing and the experts'
products, in float64 NumPy straight from the definitions. It shares no code with the CUDA path.

Rounding points are the definitions' own: the residual sum is rounded to the model's dtype, MX
blocks are rounded to e4m3 with a power-of-two scale, and everything else stays in float64.
"""
from __future__ import annotations

import numpy as np

BLOCK = 32
E4M3_MAX = 448.0


def round_bf16(a):
    """Nearest bfloat16 (ties to even) of finite values, as float64; non-finite values stay."""
    f = np.asarray(a, np.float64)
    with np.errstate(invalid="ignore"):
        m, e = np.frexp(f)
        step = np.ldexp(1.0, np.maximum(e - 8, -133))
        r = np.rint(f / step) * step
    return np.where(np.isfinite(f), r, f)


def e4m3(v):
    """Nearest e4m3 value (ties to even) of values up to 448 in magnitude."""
    v = np.asarray(v, np.float64)
    _, e = np.frexp(v)
    step = np.ldexp(1.0, np.maximum(e - 1, -6) - 3)  # 3 fraction bits; 2^-9 below 2^-6
    return np.rint(v / step) * step


def mx_scale_exponent(top):
    """Smallest e >= -127 with top * 2^-e <= 448, by search from below the answer."""
    top = np.asarray(top, np.float64)
    _, x = np.frexp(top)
    e = np.maximum(np.where(top > 0, x - 12, -127), -127).astype(int)
    for _ in range(12):
        e = np.where(top > E4M3_MAX * np.ldexp(1.0, e), e + 1, e)
    return e


def mx_round(v):
    """(code values, scale bytes) of rows [..., n]; a block with a NaN or an infinity: NaN codes
    and byte 255."""
    v = np.asarray(v, np.float64)
    blocks = v.reshape(*v.shape[:-1], v.shape[-1] // BLOCK, BLOCK)
    bad = ~np.isfinite(blocks).all(-1)
    safe = np.where(bad[..., None], 0.0, blocks)
    e = mx_scale_exponent(np.abs(safe).max(-1))
    codes = e4m3(safe * np.ldexp(1.0, -e)[..., None])
    codes = np.where(bad[..., None], np.nan, codes).reshape(v.shape)
    return codes, np.where(bad, 255, e + 127).astype(np.uint8)


def mx_value(codes, scale_bytes):
    s = np.ldexp(1.0, scale_bytes.astype(int) - 127)
    return np.asarray(codes, np.float64) * np.repeat(s, BLOCK, -1)


def tile_scales(s):
    """Scale bytes [rows, blocks] in tiles of 128 rows by 4 blocks, written byte by byte."""
    rows, blocks = s.shape
    out = np.zeros((-(-rows // 128), -(-blocks // 4), 512), np.uint8)
    for r in range(rows):
        for c in range(blocks):
            out[r // 128, c // 4, r % 32 * 16 + r % 128 // 32 * 4 + c % 4] = s[r, c]
    return out


def residual_norm(x, delta, weight, eps, bf16):
    """(r, n): the sum rounded to the dtype (fp32 addition, then bf16), and the norm unrounded."""
    r = np.asarray(x, np.float32)
    if delta is not None:
        r = r + np.asarray(delta, np.float32)
    r = round_bf16(r) if bf16 else r.astype(np.float64)
    with np.errstate(invalid="ignore", over="ignore"):
        n = r / np.sqrt((r * r).mean(-1, keepdims=True) + eps)
    if weight is not None:
        n = n * np.asarray(weight, np.float64)
    return r, n


def route(logits, top_k, scoring="softmax", bias=None, groups=1, top_groups=1, renormalise=True,
          scale=1.0):
    """(ids, weights, invalid, gap) token by token with plain loops. `gap`: the least distance
    between two different choices (or group ranks) that decide an id or an order, relative to
    them; float32 arithmetic cannot be asked to agree where it is near its own resolution."""
    t, n = logits.shape
    ids = np.full((t, top_k), -1, np.int32)
    weights = np.zeros((t, top_k))
    invalid = np.zeros(t, bool)
    gap = np.inf
    for i in range(t):
        l = np.asarray(logits[i], np.float64)
        if np.isnan(l).any() or (l == np.inf).any():
            invalid[i] = True
            continue
        on = [e for e in range(n) if l[e] > -np.inf]
        if not on:
            continue
        if scoring == "softmax":
            x = np.exp(l - l[on].max())
            score = x / x.sum()
        else:
            with np.errstate(over="ignore"):
                score = 1 / (1 + np.exp(-l))
        choice = {e: score[e] + (0.0 if bias is None else float(bias[e])) for e in on}
        if top_groups < groups:
            size = n // groups
            rank = []
            for g in range(groups):
                c = sorted((choice.get(e, -np.inf) for e in range(g * size, (g + 1) * size)),
                           reverse=True)
                rank.append(sum(c[:2]))
            order = sorted(range(groups), key=lambda g: (-rank[g], g))
            a, b = rank[order[top_groups - 1]], rank[order[top_groups]]
            if a != b and np.isfinite(a) and np.isfinite(b):
                gap = min(gap, (a - b) / max(abs(a), abs(b)))
            kept = set(order[:top_groups])
            choice = {e: c for e, c in choice.items() if e // size in kept}
        order = sorted(choice, key=lambda e: (-choice[e], e))
        for a, b in zip(order[:top_k], order[1:top_k + 1]):
            if choice[a] != choice[b]:
                gap = min(gap, (choice[a] - choice[b]) / max(abs(choice[a]), abs(choice[b])))
        chosen = order[:top_k]
        ids[i, :len(chosen)] = chosen
        w = score[chosen]
        if renormalise:
            w = w / w.sum() if w.sum() > 0 else w * 0
        weights[i, :len(chosen)] = w * scale
    return ids, weights, invalid, gap


def plan(ids, experts):
    """(offsets, rows): the pairs of every expert in rising order, then -1 for pairs without."""
    flat = np.asarray(ids).reshape(-1)
    runs = [[i for i in range(len(flat)) if flat[i] == e] for e in range(experts)]
    offsets = np.concatenate([[0], np.cumsum([len(r) for r in runs])]).astype(np.int32)
    rows = [i for r in runs for i in r]
    return offsets, np.array(rows + [-1] * (len(flat) - len(rows)), np.int32)


def experts(x, w1, w3, w2, ids, weights, mx, accumulate=2.0 ** -20):
    """(y, tolerance) for values x [tokens, dim], w1, w3 [experts, hidden, dim], w2 [experts,
    dim, hidden]. mx: h is rounded to MXFP8, else to bf16.

    The tolerance bounds what fp32 arithmetic may change, element by element. A sum of products
    kept in fp32 is off by at most `accumulate` times the sum of the products' magnitudes.
    With g and u off by their bounds, h is off by 1.1 |u| dg + |silu(g)| du (silu's slope is
    below 1.1) and 2^-20 of itself for the exponential and the division (an exponential whose
    error grows with |g|, as the hardware's does, leaves that below g = -13, where silu is so small
    that the first term covers it: dg is at least 2^-20 |g|); its rounding then gives a value
    between the roundings of h's two ends. Through w2, those differences, the sum's own bound, and
    the routing weights."""
    t, k = ids.shape
    y = np.zeros((t, x.shape[1]))
    tol = np.zeros_like(y)

    def rounded(h):
        return mx_value(*mx_round(h)) if mx else round_bf16(h)

    for i in range(t):
        for s in range(k):
            e = ids[i, s]
            if e < 0:
                continue
            with np.errstate(over="ignore", invalid="ignore"):
                g, u = w1[e] @ x[i], w3[e] @ x[i]
                dg = accumulate * (np.abs(w1[e]) @ np.abs(x[i]))
                du = accumulate * (np.abs(w3[e]) @ np.abs(x[i]))
                silu = g / (1 + np.exp(-g))
                h = silu * u
                dh = 1.1 * np.abs(u) * dg + np.abs(silu) * du + 2.0 ** -20 * np.abs(h)
                q = rounded(h)
                dq = np.maximum(np.abs(rounded(h + np.copysign(dh, h)) - q),
                                np.abs(rounded(h - np.copysign(dh, h)) - q))
                o = w2[e] @ q
                do = np.abs(w2[e]) @ dq + accumulate * (np.abs(w2[e]) @ np.abs(q))
            y[i] += weights[i, s] * o
            tol[i] += abs(weights[i, s]) * do
    return y, tol
