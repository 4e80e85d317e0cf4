"""The operators of decoding over a shared prefix cache, as cases to measure: what goes in, what
comes out, and a plain form of each.

Many sequences are decoded behind one prefix (a system prompt, an image, a long document) whose
keys and values are in a cache. Three operators:

* attn     one layer's attention of a step: the query rows of every sequence attend every key of
           the shared prefix and the keys of their own sequence, the latter under the state mask
           (which copy, x^j or its shadow s^j, of each block position a row sees); with the
           logarithm of each row's softmax normaliser as a second output;
* weights  the attention weight that each key of the prefix has received: per key/value head the
           sum of the probabilities over the query rows and the heads of the group, added to a
           decayed earlier sum;
* evict    per key/value head the n keys of the prefix to keep: the first and the last few, and
           of the others those with the largest weights (ties to the lowest index), moved
           together in their order.
"""
import math

import torch

own = False

M, C, U = 0, 1, 2  # states of block positions: masked, candidate, unmasked


def _dev():
    return torch.device("cuda")


def _dtype(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


# ------------------------------------------------------------------------------- cases
def listed():
    return [
        # one new token behind a cached prompt: reading the cache, and the launches
        dict(name="attn-one-token", op="attn", dtype="bf16", hq=28, hkv=4, dim=128, prefix=4096,
             seqs=1, text=1, block=0, after=0, shadow=False, cached=False, ragged=False),
        # a small fp32 model: the block and its shadow rows of three sequences
        dict(name="attn-small-fp32", op="attn", dtype="f32", hq=4, hkv=4, dim=64, prefix=333,
             seqs=3, text=0, block=32, after=0, shadow=True, cached=False, ragged=False),
        # ragged questions about one document, their own text cached too, odd sizes throughout
        dict(name="attn-odd", op="attn", dtype="bf16", hq=28, hkv=4, dim=64, prefix=2311,
             seqs=13, text=37, block=13, after=0, shadow=True, cached=True, ragged=True),
        # an image and its prompt shared by a batch: each sequence's question is cached, its block
        # and the shadow copies are the queries
        dict(name="attn-block", op="attn", dtype="bf16", hq=32, hkv=32, dim=128, prefix=704,
             seqs=32, text=128, block=32, after=0, shadow=True, cached=True, ragged=False),
        # few rows behind a very long document (a length that ends inside every tile)
        dict(name="attn-long", op="attn", dtype="bf16", hq=28, hkv=4, dim=128, prefix=65537,
             seqs=4, text=0, block=64, after=0, shadow=True, cached=False, ragged=False),
        # the largest: whole generations of a batch, block by block, behind a long prompt
        dict(name="attn-batch", op="attn", dtype="bf16", hq=28, hkv=4, dim=128, prefix=32768,
             seqs=16, text=0, block=32, after=224, shadow=True, cached=False, ragged=False),
        # the weights of one token's attention
        dict(name="weights-one-token", op="weights", dtype="bf16", hq=28, hkv=4, dim=128,
             prefix=4096, rows=1, first=False),
        # odd sizes in fp32, the first sum of a cache
        dict(name="weights-odd-fp32", op="weights", dtype="f32", hq=6, hkv=2, dim=64, prefix=1023,
             rows=77, first=True),
        # every row of a batch over a long prompt
        dict(name="weights-batch", op="weights", dtype="bf16", hq=28, hkv=4, dim=128,
             prefix=32768, rows=4608, first=False),
        # an image's keys down to the ones that are looked at
        dict(name="evict-image", op="evict", dtype="bf16", hkv=32, dim=128, prefix=704, keep=512,
             keep_first=4, keep_last=64),
        # odd sizes, an fp32 cache
        dict(name="evict-odd-fp32", op="evict", dtype="f32", hkv=3, dim=64, prefix=4099,
             keep=1111, keep_first=1, keep_last=33),
        # a long document's keys down to a quarter
        dict(name="evict-long", op="evict", dtype="bf16", hkv=32, dim=128, prefix=65537,
             keep=16385, keep_first=4, keep_last=1024),
    ]


_LARGEST_FLOPS = 4.0 * 16 * 288 * 28 * 128 * (32768 + 288)


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["attn", "attn", "weights", "evict"])
    dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
    hq, hkv = rng.choice([(28, 4), (32, 32), (32, 8), (4, 4), (16, 1), (6, 2), (9, 3), (40, 8)])
    dim = rng.choice([64, 128, 128])
    # fp32 runs on the CUDA cores, about 30 times slower than the matrix units
    most = _LARGEST_FLOPS / (1 if dtype == "bf16" else 30)
    prefix = _log(rng, 1, 131072)
    if op == "evict":
        prefix = min(prefix, 65537 * 32 * 128 // (hkv * dim) // (1 if dtype == "bf16" else 2))
        keep = rng.randint(max(1, prefix // 8), prefix)
        first = rng.randint(0, min(8, keep))
        last = rng.randint(0, min(512, keep - first))
        return dict(op=op, dtype=dtype, hkv=hkv, dim=dim, prefix=prefix, keep=keep,
                    keep_first=first, keep_last=last)
    if op == "weights":
        rows = min(_log(rng, 1, 9216), int(most / (4.0 * hq * dim * prefix)) + 1)
        return dict(op=op, dtype=dtype, hq=hq, hkv=hkv, dim=dim, prefix=prefix, rows=rows,
                    first=rng.random() < 0.3)
    block = rng.choice([0, 1, rng.randint(2, 128), 32])
    case = dict(op=op, dtype=dtype, hq=hq, hkv=hkv, dim=dim, prefix=prefix, seqs=_log(rng, 1, 64),
                text=rng.choice([0, 0, _log(rng, 1, 600)]) if block else _log(rng, 1, 600),
                block=block, after=rng.choice([0, 0, _log(rng, 1, 256)]) if block else 0,
                shadow=block > 0 and rng.random() < 0.8, cached=block > 0 and rng.random() < 0.5,
                ragged=rng.random() < 0.5)
    while work(case)["flops"] > most:
        if case["seqs"] > 1:
            case["seqs"] //= 2
        else:
            case["prefix"] = case["prefix"] // 2 + 1
    return case


def _layout(case):
    """Per sequence: original rows, block start, block length, shadow rows, first query row."""
    out = []
    for i in range(case["seqs"]):
        share = 1.0 if not case["ragged"] else 0.35 + 1.3 * ((i * 0.618034) % 1.0)
        text = math.ceil(case["text"] * share)
        after = math.ceil(case["after"] * share)
        b = case["block"]
        s = 0 if not case["shadow"] else b if not case["ragged"] else max(1, b - i % 3)
        out.append((text + b + after, text, b, s, text if case["cached"] else 0))
    return out


# ------------------------------------------------------------------------------ inputs
def _cache(rn, g, case):
    """Keys and values of the prefix [prefix, hkv, dim]: a few keys stand out."""
    p, hkv, d = case["prefix"], case["hkv"], case["dim"]
    k = rn(p, hkv, d)
    k *= torch.exp(0.3 * rn(p, hkv, 1))
    return k.to(_dtype(case)), rn(p, hkv, d).to(_dtype(case))


def prepare(case, seed):
    g = torch.Generator(device=_dev()).manual_seed(seed)
    op, dev, s, dt = case["op"], _dev(), dict(case), _dtype(case)

    def rn(*shape):
        return torch.randn(*shape, generator=g, device=dev, dtype=torch.float32)

    s["prefix_k"], s["prefix_v"] = _cache(rn, g, case)
    p, hkv, d = case["prefix"], case["hkv"], case["dim"]
    if op == "attn":
        lay = _layout(case)
        n, b0, b, sh, qs = ([x[j] for x in lay] for j in range(5))
        rows, hq = sum(n) + sum(sh), case["hq"]
        s["layout"] = lay
        s["q"] = (1.4 * rn(rows, hq, d)).to(dt)
        s["k"], s["v"] = rn(rows, hkv, d).to(dt), rn(rows, hkv, d).to(dt)
        nb = max(1, sum(b))
        s["state"] = torch.randint(0, 3, (nb,), generator=g, device=dev, dtype=torch.uint8)
        s["conf"] = torch.rand(nb, generator=g, device=dev)
        # shadow rows of the first positions of each block, in order
        src = [b0[i] + j for i in range(len(lay)) for j in range(sh[i])]
        s["src"] = torch.tensor(src or [0], device=dev, dtype=torch.int32)
        s["o"] = torch.zeros(rows, hq, d, device=dev, dtype=dt)
        s["lse"] = torch.zeros(rows, hq, device=dev)
        if own:
            from paper_2608_26574_gb300 import binding as B
            need = B.dard_prefix_attention_workspace_size(rows, hq, hkv, d, p)
            s["call"] = B.PrefixAttentionCall(
                n, b0, b, sh, s["state"], s["conf"], s["src"], query_start=qs,
                workspace=torch.zeros(max(need, 16), device=dev, dtype=torch.uint8))
    elif op == "weights":
        rows, hq = case["rows"], case["hq"]
        s["q"] = (1.4 * rn(rows, hq, d)).to(dt)
        # normalisers as the attention leaves them: estimated from some of the keys
        some = torch.randint(0, p, (min(p, 256),), generator=g, device=dev)
        z = torch.einsum("rhgd,khd->rhgk", s["q"].float().view(rows, hkv, -1, d),
                         s["prefix_k"][some].float()) / math.sqrt(d)
        s["lse"] = (torch.logsumexp(z, -1) + math.log(p / len(some)) + 0.1).view(rows, hq)
        s["before"] = None if case["first"] else torch.rand(hkv, p, generator=g, device=dev) * (
            2.0 * rows * hq / (hkv * p))
        s["decay"] = 1.0 if case["first"] else 0.9
        if own:
            from paper_2608_26574_gb300 import binding as B
            need = B.dard_prefix_weights_workspace_size(rows, hq, hkv, d, p)
            s["call"] = B.PrefixWeightsCall(
                decay=s["decay"],
                workspace=torch.zeros(max(need, 16), device=dev, dtype=torch.uint8))
            s["weights"] = torch.empty(hkv, p, device=dev)
    else:
        # weights over many orders of magnitude; some keys were never looked at, some share a value
        w = torch.exp(2.0 * rn(hkv, p))
        w = torch.where(rn(hkv, p) < -1.2, 0.0, w)
        s["weights"] = torch.where(rn(hkv, p) > 1.2, w.to(torch.bfloat16).float(), w)
        if own:
            from paper_2608_26574_gb300 import binding as B
            n = case["keep"]
            s["call"] = B.PrefixEvictCall(keep_first=case["keep_first"],
                                          keep_last=case["keep_last"])
            s["kept"] = torch.empty(hkv, n, device=dev, dtype=torch.int32)
            s["weights_out"] = torch.empty(hkv, n, device=dev)
            s["k_out"] = torch.empty(n, hkv, d, device=dev, dtype=dt)
            s["v_out"] = torch.empty(n, hkv, d, device=dev, dtype=dt)
    return s


# ------------------------------------------------------------------------- plain forms
def _visible(lay, state, conf, src, r0):
    """Visibility [rows r0 .., rows] of one sequence's own keys for its query rows."""
    n, b0, b, sh, _ = lay
    dev = state.device
    r = torch.arange(r0, n + sh, device=dev)
    pos = r.clone()  # the position that a row stands for
    pos[r >= n] = src.long()[r[r >= n] - n]
    qs = r >= n
    j = pos - b0
    inside = (j >= 0) & (j < b)
    jc = j.clamp(0, max(b - 1, 0))
    see = torch.ones(len(r), n + sh, dtype=torch.bool, device=dev)
    if b == 0:
        return see
    qst = torch.where(inside, state.long()[jc], torch.where(pos < b0, U, M))[:, None]
    qcf = torch.where(inside, conf[jc], 0.0)[:, None]
    same = (j[:, None] == torch.arange(b, device=dev)[None]) & qs[:, None]
    shadow = qs[:, None]
    kst, kcf = state.long()[None], conf[None]
    takes = torch.where(
        kst == U, same,
        torch.where(kst == M, shadow | (qst != M),
                    torch.where(qst == M, shadow,
                                torch.where(qst == U, True, ~(qcf <= kcf) | same))))
    has = torch.zeros(b, dtype=torch.bool, device=dev)
    at = src.long() - b0
    has[at] = True
    see[:, b0:b0 + b] = ~(takes & has[None])
    see[:, n:] = takes[:, at]
    return see


def _sequences(s):
    """(layout, first row, state, conf, shadow sources) of each sequence."""
    row = blk = sh = 0
    for lay in s["layout"]:
        n, _, b, z, _ = lay
        yield lay, row, s["state"][blk:blk + b], s["conf"][blk:blk + b], s["src"][sh:sh + z]
        row, blk, sh = row + n + z, blk + b, sh + z


def _plain_attn(s):
    hq, hkv, d, p = s["hq"], s["hkv"], s["dim"], s["prefix"]
    g, scale = hq // hkv, 1 / math.sqrt(d)
    o, lse = torch.zeros_like(s["o"]), torch.zeros_like(s["lse"])
    pk, pv = s["prefix_k"].float().transpose(0, 1), s["prefix_v"].float().transpose(0, 1)
    for lay, row, state, conf, src in _sequences(s):
        n, _, _, sh, qs = lay
        see = _visible(lay, state, conf, src, qs)
        k, v = (s[x][row:row + n + sh].float().transpose(0, 1) for x in ("k", "v"))
        q = s["q"][row + qs:row + n + sh].float()
        rq = q.shape[0]
        q = q.view(rq, hkv, g, d).permute(1, 2, 0, 3)  # [hkv, g, rows, d]
        step = max(1, (1 << 28) // (g * rq * (p + n + sh)))  # heads at a time
        for h in range(0, hkv, step):
            kk = torch.cat([pk[h:h + step], k[h:h + step]], 1)
            vv = torch.cat([pv[h:h + step], v[h:h + step]], 1)
            hs = kk.shape[0]
            z = (q[h:h + step].reshape(hs, g * rq, d) @ kk.mT).view(hs, g, rq, -1) * scale
            z[..., p:].masked_fill_(~see, -math.inf)
            top = z.amax(-1, keepdim=True)
            e = torch.exp(z - top)
            total = e.sum(-1, keepdim=True)
            out = (e.view(hs, g * rq, -1) @ vv).view(hs, g, rq, d) / total
            heads = slice(h * g, (h + hs) * g)
            rows = slice(row + qs, row + n + sh)
            o[rows, heads] = out.permute(2, 0, 1, 3).reshape(rq, hs * g, d).to(o.dtype)
            lse[rows, heads] = (top + torch.log(total))[..., 0].permute(2, 0, 1).reshape(rq, hs * g)
    return {"o": o, "lse": lse}


def _plain_weights(s):
    hq, hkv, d, p, rows = s["hq"], s["hkv"], s["dim"], s["prefix"], s["rows"]
    g, scale = hq // hkv, 1 / math.sqrt(d)
    q = s["q"].float().view(rows, hkv, g, d).permute(1, 0, 2, 3).reshape(hkv, rows * g, d)
    lse = s["lse"].view(rows, hkv, g).permute(1, 0, 2).reshape(hkv, rows * g, 1)
    k = s["prefix_k"].float().transpose(0, 1)
    w = torch.zeros(hkv, p, device=q.device) if s["before"] is None else s["decay"] * s["before"]
    step = max(1, (1 << 28) // (rows * g * hkv))  # keys at a time
    for at in range(0, p, step):
        z = q @ k[:, at:at + step].mT * scale
        w[:, at:at + step] += torch.exp(z - lse).sum(1)
    return {"weights": w}


def _plain_evict(s):
    w, p, n = s["weights"], s["prefix"], s["keep"]
    first, last = s["keep_first"], s["keep_last"]
    middle = w[:, first:p - last]
    order = torch.sort(middle, dim=-1, descending=True, stable=True).indices
    chosen = torch.sort(order[:, :n - first - last], dim=-1).values + first
    heads = torch.arange(w.shape[0], device=w.device)[:, None]
    ends = torch.cat([torch.arange(first, device=w.device),
                      torch.arange(p - last, p, device=w.device)]).expand(w.shape[0], -1)
    kept = torch.cat([ends[:, :first], chosen, ends[:, first:]], 1)
    k, v = (s[x][kept, heads].transpose(0, 1).contiguous() for x in ("prefix_k", "prefix_v"))
    return {"kept": kept.to(torch.int32), "k": k, "v": v, "weights": w.gather(1, kept)}


# --------------------------------------------------------------------------- one pass
def run(state):
    s = state
    if not own:
        return {"attn": _plain_attn, "weights": _plain_weights, "evict": _plain_evict}[s["op"]](s)
    if s["op"] == "attn":
        s["call"](s["q"], s["k"], s["v"], s["o"], s["prefix_k"], s["prefix_v"], lse=s["lse"])
        return {"o": s["o"], "lse": s["lse"]}
    if s["op"] == "weights":
        s["call"](s["q"], s["lse"], s["prefix_k"], s["weights"], weights_in=s["before"])
        return {"weights": s["weights"]}
    s["call"](s["weights"], s["prefix_k"], s["prefix_v"], s["kept"], s["k_out"], s["v_out"],
              weights_out=s["weights_out"])
    return {"kept": s["kept"], "k": s["k_out"], "v": s["v_out"], "weights": s["weights_out"]}


def work(case):
    d, p, hkv, z = case["dim"], case["prefix"], case["hkv"], 2 if case["dtype"] == "bf16" else 4
    if case["op"] == "evict":
        n = case["keep"]
        return {"bytes": hkv * (4 * p + 8 * n) + 4 * n * hkv * d * z, "flops": hkv * p}
    hq = case["hq"]
    if case["op"] == "weights":
        r = case["rows"]
        return {"bytes": r * hq * (d * z + 4) + p * hkv * (d * z + (4 if case["first"] else 8)),
                "flops": 2.0 * r * hq * p * d}
    lay = _layout(case)
    queries = sum(n + s - qs for n, _, _, s, qs in lay)
    keys = sum(n + s for n, _, _, s, _ in lay)
    # every query attends the prefix and one copy of each position of its sequence
    pairs = sum((n + s - qs) * (p + n) for n, _, _, s, qs in lay)
    return {"bytes": queries * hq * (2 * d * z + 4) + 2 * (keys + p) * hkv * d * z,
            "flops": 4.0 * pairs * hq * d}


# ---------------------------------------------------------------------- in 64 bits
# The copy of a key position that a query takes, by the states of the key and of the query:
# 0 = x, 1 = s, 2 = s where the query's confidence is above the key's.
_ORIGINAL = {M: {M: 0, C: 1, U: 1}, C: {M: 0, C: 2, U: 1}, U: {M: 0, C: 0, U: 0}}
_SHADOW = {M: {M: 1, C: 1, U: 1}, C: {M: 1, C: 2, U: 1}, U: {M: 0, C: 0, U: 0}}


def _seen(lay, state, conf, src):
    """Rows x rows visibility of one sequence, position by position of its block."""
    n, b0, b, sh, _ = lay
    st, cf, at = state.tolist(), conf.double().tolist(), [x - b0 for x in src.tolist()[:sh]]
    state_of = [U] * b0 + st + [M] * (n - b0 - b)
    see = torch.zeros(n + sh, n + sh, dtype=torch.bool)
    see[:, :n] = True
    for k, j in enumerate(at):
        rule = torch.tensor([[t[st[j]][q] for q in (M, C, U)] for t in (_ORIGINAL, _SHADOW)])
        queries = torch.tensor(state_of + [st[i] for i in at])
        copy = torch.tensor([0] * n + [1] * sh)
        mine = torch.tensor([0.0] * b0 + cf + [0.0] * (n - b0 - b) + [cf[i] for i in at],
                            dtype=torch.float64)
        choice = rule[copy, queries]
        take = (choice == 1) | ((choice == 2) & (mine > cf[j]))
        take[n + k] = True  # a shadow row always sees itself
        see[:, b0 + j] = ~take
        see[:, n + k] = take
    return see.to(_dev())


def exact(case, seed):
    s, op = prepare(case, seed), case["op"]
    d, p, hkv = case["dim"], case["prefix"], case["hkv"]
    if op == "evict":
        w, n = s["weights"].double().cpu(), case["keep"]
        first, last = case["keep_first"], case["keep_last"]
        rank = w.clone()
        rank[:, :first] = math.inf
        rank[:, p - last:] = math.inf
        # a stable sort of the negated weights: equal weights stay in rising order
        kept = torch.argsort(-rank, dim=1, stable=True)[:, :n].sort(1).values.to(_dev())
        pick = [s[x].transpose(0, 1).double().gather(1, kept[..., None].expand(-1, -1, d))
                .transpose(0, 1) for x in ("prefix_k", "prefix_v")]
        return {"kept": None, "k": pick[0], "v": pick[1],
                "weights": s["weights"].double().gather(1, kept)}
    if work(case)["flops"] > 8e12:
        return None
    hq = case["hq"]
    g = hq // hkv
    if op == "weights":
        out = torch.zeros(hkv, p, dtype=torch.float64, device=_dev())
        step = max(1, (1 << 26) // p)
        for h in range(hq):
            key = s["prefix_k"][:, h // g].double()
            for r in range(0, case["rows"], step):
                z = torch.einsum("rd,kd->rk", s["q"][r:r + step, h].double(), key) / d ** 0.5
                out[h // g] += torch.exp(z - s["lse"][r:r + step, h, None].double()).sum(0)
        if s["before"] is not None:
            out += s["before"].double() * s["decay"]
        return {"weights": out}
    o = torch.zeros(s["o"].shape, dtype=torch.float64, device=_dev())
    lse = torch.zeros(s["lse"].shape, dtype=torch.float64, device=_dev())
    for lay, row, state, conf, src in _sequences(s):
        n, _, _, sh, qs = lay
        see = _seen(lay, state, conf, src)
        own_rows = slice(row, row + n + sh)
        for h in range(hq):
            key = torch.cat([s["prefix_k"][:, h // g], s["k"][own_rows, h // g]]).double()
            val = torch.cat([s["prefix_v"][:, h // g], s["v"][own_rows, h // g]]).double()
            step = max(1, (1 << 26) // len(key))
            for r in range(qs, n + sh, step):
                at = slice(row + r, row + min(r + step, n + sh))
                z = s["q"][at, h].double() @ key.T / d ** 0.5
                z[:, p:][~see[r:r + step]] = -math.inf
                lse[at, h] = torch.logsumexp(z, 1)
                o[at, h] = torch.softmax(z, 1) @ val
    return {"o": o, "lse": lse}
