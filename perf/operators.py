"""The operators of a mixture-of-experts MLP in microscaled 8-bit floating point (MXFP8), as
cases to measure: what goes in, what comes out, and a plain form of each.

Four operators, in the order in which one layer runs them:

* norm      the residual addition, the root-mean-square norm of the sum, and its rounding to
            e4m3 codes with one power-of-two scale for each 32 elements of a row;
* quantize  the same rounding alone: activations (scales by rows) and weights (scales in the
            tiles of 128 rows by 4 scales that the matrix instruction reads);
* route     scores of every expert, groups, top-k, renormalised weights, and the plan: the
            (token, slot) pairs sorted by expert;
* experts   for every (token, slot) pair W2 (silu(W1 x) * (W3 x)) of its expert, the product
            in between rounded to MXFP8 too, and the weighted sum over a token's slots.

The MX rounding: a block of 32 values has the scale 2^e with the smallest e for which
max|v| 2^-e <= 448 (the largest e4m3 value), at least 2^-127; codes are v 2^-e rounded to the
nearest even e4m3 value; the scale is kept as the byte e + 127 (e8m0).
"""
import math

import torch

own = False

MX = 32


def _dev():
    return torch.device("cuda")


def _dtype(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


def _up(n, to):
    return -(-n // to) * to


# ------------------------------------------------------------------------------- cases
def listed():
    return [
        # one token of a dense layer (the 8B-shaped model's width) between attention and MLP
        dict(name="norm-one-token", op="norm", tokens=1, dim=4096, dtype="bf16", delta=True,
             weight=True, keep=True, mx=True, pad=0),
        # an fp32 model of an odd width, rows inside a wider buffer, no 8-bit output
        dict(name="norm-odd-fp32", op="norm", tokens=1777, dim=2731, dtype="f32", delta=True,
             weight=True, keep=True, mx=False, pad=13),
        # the rows of a whole batch of ragged prompts
        dict(name="norm-batch", op="norm", tokens=38912, dim=4096, dtype="bf16", delta=True,
             weight=True, keep=True, mx=True, pad=0),
        # the rows of one block and its shadow copies, an odd number of 32-element blocks
        dict(name="quantize-block", op="quantize", batch=1, rows=65, dim=2080, dtype="f32",
             tiles=False),
        # loading a layer: the weights of 64 experts, laid out for the product
        dict(name="quantize-weights", op="quantize", batch=64, rows=2048, dim=2048,
             dtype="bf16", tiles=True),
        # one token
        dict(name="route-one-token", op="route", tokens=1, experts=64, top_k=8, dtype="bf16",
             scoring="softmax", groups=1, top_groups=1, bias=False, masked=False),
        # a batch of prompts with groups of experts and a bias, some experts switched off
        dict(name="route-groups", op="route", tokens=5121, experts=160, top_k=6, dtype="f32",
             scoring="sigmoid", groups=8, top_groups=3, bias=True, masked=True),
        # the largest: many prompts at once
        dict(name="route-batch", op="route", tokens=38912, experts=256, top_k=8, dtype="f32",
             scoring="sigmoid", groups=8, top_groups=4, bias=True, masked=False),
        # one token through eight experts: the weights' bytes and the launches
        dict(name="experts-one-token", op="experts", tokens=1, experts=64, top_k=8, dim=2048,
             hidden=1024),
        # ragged experts of odd widths, some rows without a full set of experts
        dict(name="experts-odd", op="experts", tokens=1111, experts=40, top_k=6, dim=2208,
             hidden=736),
        # one expert: the dense MLP of the decoding example, one augmented sequence
        dict(name="experts-dense", op="experts", tokens=800, experts=1, top_k=1, dim=4096,
             hidden=12288),
        # the largest: a batch of prompts through 64 experts
        dict(name="experts-batch", op="experts", tokens=8192, experts=64, top_k=8, dim=4096,
             hidden=2048),
    ]


def _log(rng, lo, hi):
    n = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    return n - 1 if n == 3072 else n


def _width(rng, lo, hi):
    return min(32 * _log(rng, lo, hi), 32 * hi) // 96 * 96 + rng.choice([32, 64, 128])


def draw(rng):
    op = rng.choice(["norm", "quantize", "route", "experts"])
    if op == "norm":
        mx = rng.random() < 0.6
        dim = _width(rng, 8, 250) if mx else _log(rng, 100, 8192)
        dtype = rng.choice(["bf16", "bf16", "f32"])
        most = 38912 * 4096 // (dim if dtype == "bf16" else 2 * dim)
        return dict(op=op, tokens=_log(rng, 1, min(38912, most)), dim=dim, dtype=dtype,
                    delta=rng.random() < 0.75, weight=rng.random() < 0.75,
                    keep=rng.random() < 0.75 or not mx, mx=mx, pad=rng.choice([0, 0, 8, 5]))
    if op == "quantize":
        dim = _width(rng, 2, 250)
        batch = rng.choice([1, 1, _log(rng, 2, 64)])
        dtype = rng.choice(["bf16", "f32"])
        most = 64 * 2048 * 2048 // (batch * dim) // (1 if dtype == "bf16" else 2)
        return dict(op=op, batch=batch, rows=_log(rng, 1, min(8192, most)), dim=dim, dtype=dtype,
                    tiles=rng.random() < 0.5)
    if op == "route":
        groups = rng.choice([1, 1, 4, 8])
        experts = groups * rng.randint(max(2, 16 // groups), 256 // groups)
        top_groups = rng.randint(max(1, groups // 4), groups)
        top_k = rng.randint(1, min(12, top_groups * (experts // groups)))
        scoring = "sigmoid" if groups > 1 else rng.choice(["softmax", "sigmoid"])
        return dict(op=op, tokens=_log(rng, 1, 38912), experts=experts, top_k=top_k,
                    dtype=rng.choice(["bf16", "f32"]), scoring=scoring, groups=groups,
                    top_groups=top_groups, bias=scoring == "sigmoid" and rng.random() < 0.7,
                    masked=rng.random() < 0.3)
    experts = rng.choice([1, _log(rng, 4, 128), _log(rng, 4, 128)])
    top_k = rng.randint(1, min(8, experts))
    dim, hidden = _width(rng, 16, 124), _width(rng, 8, 380)
    while experts * dim * hidden > 64 * 4096 * 2048:
        experts = max(top_k, experts // 2)
        hidden = max(320, hidden // 192 * 96 + 32)
    most = 8192 * 8 * 4096 * 2048 // (top_k * dim * hidden)
    return dict(op=op, tokens=_log(rng, 1, min(8192, most)), experts=experts, top_k=top_k,
                dim=dim, hidden=hidden)


# ------------------------------------------------------------------------------ inputs
def _codes(g, *shape):
    """e4m3 codes as a quantised normal variable has them: up to 448, about 2.3 deviations."""
    return (torch.randn(*shape, generator=g, device=_dev(), dtype=torch.bfloat16) * 110.0) \
        .clamp_(-448, 448).to(torch.float8_e4m3fn)


def _scale_bytes(g, value_std, *shape):
    """Scales (bytes e + 127) under which those codes have about the deviation `value_std`."""
    e = 127 + math.floor(math.log2(value_std / 110.0))
    return torch.randint(e, e + 2, shape, generator=g, device=_dev(), dtype=torch.uint8)


def _plan(ids, experts):
    """(offsets, rows) of the sorted (token, slot) pairs: what the routing operator gives."""
    flat = ids.reshape(-1).long()
    key = torch.where(flat < 0, experts, flat)
    order = torch.sort(key, stable=True)
    ends = torch.searchsorted(order.values, torch.arange(experts + 1, device=ids.device))
    at = torch.arange(flat.numel(), device=ids.device)
    return (ends.to(torch.int32),
            torch.where(at < ends[experts], order.indices, -1).to(torch.int32))


def prepare(case, seed):
    g = torch.Generator(device=_dev()).manual_seed(seed)
    op, dev, s = case["op"], _dev(), dict(case)

    def rn(*shape, dtype=torch.float32):
        return torch.randn(*shape, generator=g, device=dev, dtype=torch.float32).to(dtype)

    if op == "norm":
        t, d, pad, dt = case["tokens"], case["dim"], case["pad"], _dtype(case)
        # a residual stream: a few channels far larger than the rest
        channel = torch.exp(0.7 * rn(d))
        s["x"] = (rn(t, d + pad) * torch.nn.functional.pad(channel, (0, pad))).to(dt)[:, :d]
        s["delta"] = rn(t, d + pad, dtype=dt)[:, :d] if case["delta"] else None
        s["weight"] = (1 + 0.1 * rn(d)).to(dt) if case["weight"] else None
        if own:
            from paper_2608_26574_gb300 import binding as B
            s["call"] = B.NormCall(d, dt, weight=s["weight"], eps=1e-6)
            s["residual"] = torch.empty(t, d, device=dev, dtype=dt) if case["delta"] else None
            s["y"] = torch.empty(t, d, device=dev, dtype=dt) if case["keep"] else None
            if case["mx"]:
                s["y8"] = torch.empty(t, d, device=dev, dtype=torch.float8_e4m3fn)
                s["y8_scale"] = torch.zeros(B.mx_scale_shape((t, d)), device=dev,
                                            dtype=torch.uint8)
    elif op == "quantize":
        b, r, d, dt = case["batch"], case["rows"], case["dim"], _dtype(case)
        s["x"] = rn(b, r, d, dtype=dt) * torch.exp(0.5 * rn(b, r, 1)).to(dt)
        if own:
            from paper_2608_26574_gb300 import binding as B
            layout = B.MX_SCALE_TILES if case["tiles"] else B.MX_SCALE_ROWS
            s["layout"] = layout
            s["codes"] = torch.empty(b, r, d, device=dev, dtype=torch.float8_e4m3fn)
            s["scales"] = torch.zeros(B.mx_scale_shape((b, r, d), layout), device=dev,
                                      dtype=torch.uint8)
    elif op == "route":
        t, e, k = case["tokens"], case["experts"], case["top_k"]
        # some experts are liked more than others
        s["logits"] = (rn(t, e) + 0.5 * rn(e)).to(_dtype(case))
        if case["masked"]:  # an eighth of the experts is off
            off = torch.randperm(e, generator=g, device=dev)[:e // 8]
            s["logits"][:, off] = -math.inf
        s["bias"] = 0.05 * rn(e) if case["bias"] else None
        s["scale"] = 2.5 if case["scoring"] == "sigmoid" else 1.0
        if own:
            from paper_2608_26574_gb300 import binding as B
            need = B.dard_route_workspace_size(t, e, k)
            s["call"] = B.RouteCall(
                e, k, scoring=B.ROUTE_SIGMOID if case["scoring"] == "sigmoid" else B.ROUTE_SOFTMAX,
                bias=s["bias"], groups=case["groups"], top_groups=case["top_groups"],
                renormalise=True, scale=s["scale"],
                workspace=torch.zeros(max(need, 16), device=dev, dtype=torch.uint8))
            s["ids"] = torch.empty(t, k, device=dev, dtype=torch.int32)
            s["weights"] = torch.empty(t, k, device=dev)
            s["offsets"] = torch.empty(e + 1, device=dev, dtype=torch.int32)
            s["rows"] = torch.empty(t * k, device=dev, dtype=torch.int32)
    else:
        t, e, k, d, f = (case[n] for n in ("tokens", "experts", "top_k", "dim", "hidden"))
        s["x"], s["x_scale"] = _codes(g, t, d), _scale_bytes(g, 1.0, t, _up(d // MX, 16))
        for n, r, c in (("w1", f, d), ("w3", f, d), ("w2", d, f)):
            s[n] = _codes(g, e, r, c)
            s[n + "_scale"] = _scale_bytes(g, 1 / math.sqrt(c), e, _up(r, 128) // 128,
                                           _up(c, 128) // 128, 512)
        liked = rn(t, e) + 0.3 * rn(e)
        ids = torch.topk(liked, k).indices.to(torch.int32)
        if k > 1:  # one token in 16 has a slot without an expert
            ids[:, k - 1] = torch.where(rn(t) < -1.53, -1, ids[:, k - 1])
        s["ids"], s["weights"] = ids, torch.softmax(rn(t, k), -1)
        s["offsets"], s["rows"] = _plan(ids, e)
        if own:
            from paper_2608_26574_gb300 import binding as B
            need = B.dard_experts_workspace_size(t, e, k, d, f)
            s["call"] = B.ExpertsCall(
                *(s[n + x] for n in ("w1", "w3", "w2") for x in ("", "_scale")),
                workspace=torch.empty(max(need, 16), device=dev, dtype=torch.uint8))
            s["y"] = torch.empty(t, d, device=dev, dtype=torch.bfloat16)
    return s


# ------------------------------------------------------------------------- plain forms
def _mx(v):
    """(codes, scale bytes) of the fp32 values v [..., n], a scale for each 32."""
    v = v.unflatten(-1, (-1, MX))
    m, ex = torch.frexp(v.abs().amax(-1))
    e = torch.where(m > 0.875, ex - 8, ex - 9)
    e = torch.where(m == 0, -127, e).clamp(min=-127)
    inv = ((127 - e) << 23).view(torch.float32)  # 2^-e, exactly
    codes = (v * inv[..., None]).to(torch.float8_e4m3fn)
    return codes.flatten(-2), (e + 127).to(torch.uint8)


def _pow2(scale_byte):
    b = scale_byte.int()
    return torch.where(b == 0, 2.0 ** -127, (b << 23).view(torch.float32))


def _value(codes, scale_byte):
    """codes [..., n] and scale bytes [..., n / 32] as fp32 values."""
    return (codes.float().unflatten(-1, (-1, MX)) * _pow2(scale_byte)[..., None]).flatten(-2)


def _tiled(s):
    """Scale bytes [b, rows, blocks] in tiles of 128 rows x 4 blocks: the byte of row r and
    block c of a tile is at (r % 32) * 16 + (r / 32) * 4 + c."""
    b, r, c = s.shape
    s = torch.nn.functional.pad(s, (0, _up(c, 4) - c, 0, _up(r, 128) - r))
    s = s.view(b, -1, 4, 32, s.shape[2] // 4, 4)  # tile row, r / 32, r % 32, tile column, c
    return s.permute(0, 1, 4, 3, 2, 5).reshape(b, s.shape[1], s.shape[4], 512)


def _untiled(s, rows, blocks):
    b, tr, tc, _ = s.shape
    s = s.view(b, tr, tc, 32, 4, 4).permute(0, 1, 4, 3, 2, 5).reshape(b, tr * 128, tc * 4)
    return s[:, :rows, :blocks]


def _out8(codes, scale):
    return {"codes": codes, "scale": scale.view(torch.float8_e8m0fnu)}


def _plain_norm(s):
    r = s["x"]
    if s["delta"] is not None:
        r = (r.float() + s["delta"].float()).to(r.dtype)
    f = r.float()
    y = f * torch.rsqrt((f * f).mean(-1, keepdim=True) + 1e-6)
    if s["weight"] is not None:
        y = y * s["weight"].float()
    out = {"residual": r} if s["delta"] is not None else {}
    if s["keep"]:
        out["y"] = y.to(r.dtype)
    if s["mx"]:
        out |= _out8(*_mx(y))
    return out


def _plain_quantize(s):
    codes, scale = _mx(s["x"].float())
    return _out8(codes, _tiled(scale) if s["tiles"] else scale)


def _plain_route(s):
    x, e, k, groups = s["logits"].float(), s["experts"], s["top_k"], s["groups"]
    t = x.shape[0]
    if s["scoring"] == "softmax":
        ex = torch.exp(x - x.amax(-1, keepdim=True))
        score, sel = ex / ex.sum(-1, keepdim=True), ex  # the same order before the division
    else:
        score = 1 / (1 + torch.exp(-x))
        sel = score if s["bias"] is None else score + s["bias"]
    sel = sel.masked_fill(x == -math.inf, -math.inf)
    if s["top_groups"] < groups:
        in_group = torch.sort(sel.view(t, groups, -1), -1, descending=True).values
        rank = in_group[..., :2].sum(-1)  # its two best
        kept = torch.sort(rank, dim=-1, descending=True, stable=True).indices[:, :s["top_groups"]]
        keep = torch.zeros(t, groups, dtype=torch.bool, device=x.device).scatter_(1, kept, True)
        sel = sel.masked_fill(~keep.repeat_interleave(e // groups, 1), -math.inf)
    best = torch.sort(sel, dim=-1, descending=True, stable=True)
    off = best.values[:, :k] == -math.inf
    ids = best.indices[:, :k]
    w = score.gather(1, ids).masked_fill(off, 0.0)
    total = w.sum(-1, keepdim=True)
    w = torch.where(total > 0, w / total, 0.0) * s["scale"]
    ids = ids.masked_fill(off, -1).to(torch.int32)
    offsets, rows = _plan(ids, e)
    return {"ids": ids, "weights": w, "offsets": offsets, "rows": rows}


def _mlp(x, w1, w3, w2):
    gate, up = x @ w1.mT, x @ w3.mT
    h = gate / (1 + torch.exp(-gate)) * up
    return _value(*_mx(h)) @ w2.mT


def _plain_experts(s):
    t, e, k, d, f = (s[n] for n in ("tokens", "experts", "top_k", "dim", "hidden"))
    x = _value(s["x"], s["x_scale"][:, :d // MX])
    if t * k <= e:  # few pairs: each with its own expert's weights
        which = s["ids"].reshape(-1).clamp(min=0).long()
        w = [_value(s[n][which], _untiled(s[n + "_scale"][which], r, c // MX))
             for n, r, c in (("w1", f, d), ("w3", f, d), ("w2", d, f))]
        o = _mlp(x.repeat_interleave(k, 0)[:, None], *w)[:, 0]
        o = o.masked_fill(s["ids"].reshape(-1, 1) < 0, 0.0)
    else:  # every expert's rows, padded to the most that one has
        w = [_value(s[n], _untiled(s[n + "_scale"], r, c // MX))
             for n, r, c in (("w1", f, d), ("w3", f, d), ("w2", d, f))]
        first, last = s["offsets"][:-1].long(), s["offsets"][1:].long()
        at = first[:, None] + torch.arange(int((last - first).max()), device=x.device)
        used = at < last[:, None]
        pair = s["rows"].long()[at.clamp(max=t * k - 1)].clamp(min=0)
        out = _mlp(x[pair // k], *w)
        o = torch.zeros(t * k + 1, d, device=x.device)
        o[torch.where(used, pair, t * k)] = out
        o = o[:-1]
    y = (o.view(t, k, d) * s["weights"][..., None]).sum(1)
    return {"y": y.to(torch.bfloat16)}


_PLAIN = {"norm": _plain_norm, "quantize": _plain_quantize, "route": _plain_route,
          "experts": _plain_experts}


# --------------------------------------------------------------------------- one pass
def run(state):
    s = state
    if not own:
        return _PLAIN[s["op"]](s)
    if s["op"] == "norm":
        s["call"](s["x"], s["delta"], residual=s["residual"], y=s["y"], y8=s.get("y8"),
                  y8_scale=s.get("y8_scale"))
        out = {"residual": s["residual"]} if s["delta"] is not None else {}
        if s["keep"]:
            out["y"] = s["y"]
        if s["mx"]:
            out |= _out8(s["y8"], s["y8_scale"][:, :s["dim"] // MX])
        return out
    if s["op"] == "quantize":
        from paper_2608_26574_gb300 import binding as B
        B.dard_mx_quantize(s["x"], s["codes"], s["scales"], s["layout"])
        scales = s["scales"] if s["tiles"] else s["scales"][..., :s["dim"] // MX]
        return _out8(s["codes"], scales)
    if s["op"] == "route":
        s["call"](s["logits"], s["ids"], s["weights"], s["offsets"], s["rows"])
        return {n: s[n] for n in ("ids", "weights", "offsets", "rows")}
    s["call"](s["x"], s["x_scale"], s["ids"], s["weights"], s["offsets"], s["rows"], s["y"])
    return {"y": s["y"]}


def work(case):
    op = case["op"]
    if op == "norm":
        n, z = case["tokens"] * case["dim"], 2 if case["dtype"] == "bf16" else 4
        read = n * z * (2 if case["delta"] else 1) + (case["dim"] * z if case["weight"] else 0)
        write = n * z * (case["delta"] + case["keep"]) + (n + n // MX if case["mx"] else 0)
        return {"bytes": read + write, "flops": 6 * n}
    if op == "quantize":
        n = case["batch"] * case["rows"] * case["dim"]
        return {"bytes": n * (2 if case["dtype"] == "bf16" else 4) + n + n // MX, "flops": 3 * n}
    if op == "route":
        t, e, k = case["tokens"], case["experts"], case["top_k"]
        z = 2 if case["dtype"] == "bf16" else 4
        return {"bytes": t * e * z + 4 * e * (1 + case["bias"]) + t * k * 12,
                "flops": t * e * 6}
    t, e, k, d, f = (case[n] for n in ("tokens", "experts", "top_k", "dim", "hidden"))
    used = e * (1 - (1 - k / e) ** t)  # experts that some token is sent to, on average
    weights = used * 3 * d * f * (1 + 1 / MX)
    return {"bytes": weights + t * d * (1 + 1 / MX + 2) + t * k * 12,
            "flops": 2 * t * k * 3 * d * f}


# ---------------------------------------------------------------------- in 64 bits
def _mx64(v):
    """The values that the codes and the scales stand for, from the definition."""
    blocks = v.double().reshape(*v.shape[:-1], v.shape[-1] // MX, MX)
    top = blocks.abs().max(-1, keepdim=True).values
    e = torch.ceil(torch.log2(top / 448)).nan_to_num(neginf=-127).clamp(min=-127)
    # a logarithm next to a whole number: the smallest e for which top 2^-e <= 448
    e = torch.where(top > 448 * torch.exp2(e), e + 1, e)
    e = torch.where((top <= 448 * torch.exp2(e - 1)) & (e > -127), e - 1, e)
    w = blocks / torch.exp2(e)
    # e4m3: 3 fraction bits above 2^-6, steps of 2^-9 below
    step = torch.exp2(torch.floor(torch.log2(w.abs().clamp(min=2.0 ** -6))) - 3)
    codes = (torch.round(w / step) * step).reshape(v.shape)
    return codes, torch.exp2(e)[..., 0]


def _unpack64(codes, scales, rows, blocks):
    """One expert's matrix in 64 bits from its codes and tiled scales [tr, tc, 512]."""
    r = torch.arange(rows, device=codes.device)[:, None]
    c = torch.arange(blocks, device=codes.device)[None]
    byte = scales[r // 128, c // 4, r % 32 * 16 + r % 128 // 32 * 4 + c % 4]
    return codes.double() * torch.exp2(byte.double() - 127).repeat_interleave(MX, 1)


def exact(case, seed):
    s, op = prepare(case, seed), case["op"]
    if op == "norm":
        r = s["x"].double()
        if s["delta"] is not None:
            r = (r + s["delta"].double()).to(s["x"].dtype).double()
        y = r / torch.sqrt(torch.linalg.vecdot(r, r)[:, None] / case["dim"] + 1e-6)
        y = y * s["weight"].double() if s["weight"] is not None else y
        out = {"residual": r} if s["delta"] is not None else {}
        if case["keep"]:
            out["y"] = y
        if case["mx"]:
            out["codes"], out["scale"] = _mx64(y)
        return out
    if op == "quantize":
        codes, scale = _mx64(s["x"])
        if case["tiles"]:
            b, r, c = scale.shape
            full = torch.full((b, _up(r, 128) // 128, _up(c, 4) // 4, 512), 2.0 ** -127,
                              dtype=torch.float64, device=scale.device)
            i, j = torch.arange(r, device=_dev())[:, None], torch.arange(c, device=_dev())[None]
            full[:, i // 128, j // 4, i % 32 * 16 + i % 128 // 32 * 4 + j % 4] = scale
            scale = full
        return {"codes": codes, "scale": scale}
    if op == "route":
        x = s["logits"].double()
        score = torch.softmax(x, -1) if case["scoring"] == "softmax" else torch.sigmoid(x)
        sel = score if s["bias"] is None else score + s["bias"].double()
        sel = torch.where(torch.isneginf(x), x, sel).reshape(len(x), case["groups"], -1)
        best2 = torch.topk(sel, min(2, sel.shape[-1]), -1).values.sum(-1)
        order = torch.argsort(-best2, dim=-1, stable=True)
        place = torch.argsort(order, -1)  # of each group
        sel = sel.masked_fill((place >= case["top_groups"])[..., None], -math.inf).flatten(1)
        ids = torch.argsort(-sel, dim=-1, stable=True)[:, :case["top_k"]]
        w = score.gather(1, ids) * (sel.gather(1, ids) > -math.inf)
        total = w.sum(-1, keepdim=True)
        return {"ids": None, "offsets": None, "rows": None,
                "weights": torch.where(total > 0, w / total, 0.0) * s["scale"]}
    t, e, k, d, f = (case[n] for n in ("tokens", "experts", "top_k", "dim", "hidden"))
    if 2.0 * t * k * 3 * d * f > 8e12:
        return None
    x = s["x"].double() * torch.exp2(s["x_scale"][:, :d // MX].double() - 127) \
        .repeat_interleave(MX, 1)
    y = torch.zeros(t, d, dtype=torch.float64, device=_dev())
    for i in range(e):
        token, slot = torch.nonzero(s["ids"] == i, as_tuple=True)
        if not len(token):
            continue
        w1, w3, w2 = (_unpack64(s[n][i], s[n + "_scale"][i], r, c // MX)
                      for n, r, c in (("w1", f, d), ("w3", f, d), ("w2", d, f)))
        gate = x[token] @ w1.T
        codes, scale = _mx64(gate * torch.sigmoid(gate) * (x[token] @ w3.T))
        o = (codes * scale.repeat_interleave(MX, 1)) @ w2.T
        y.index_add_(0, token, o * s["weights"][token, slot].double()[:, None])
    return {"y": y}
