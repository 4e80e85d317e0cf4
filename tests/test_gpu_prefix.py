"""Decoding behind a shared prefix on the GPU against the float64 oracle.

Tolerances, derived from the arithmetic before any run (u = 2^-24, half a step of fp32):
* A score: d products and their sum in fp32 (the tensor cores may cut instead of rounding: a whole
  step each), so it is off by at most ds = 2 (d + 4) u sum|q k| scale.
* Attention in bf16: the probabilities are rounded to bf16 (2^-8 each) and divided by the sum of the
  rounded ones: 2^-7 sum p|v|; scores and exponentials move them by 2 ds + 2^-20, n additions by
  2 n u; the output's rounding 2^-8 |o|. In fp32 without the two roundings to bf16.
* lse: ds, the exponentials' 2^-20, the additions' 2 n u, and 4 u |lse| for the logarithm's form.
* weights: every term ds + 2^-20 + 4 u |lse|, the additions at most 64 + terms / 64 in a chain.
* kept, k, v and the kept weights: equal.
"""
import math

import numpy as np
import pytest
import torch

from oracle import dard_oracle as D
from oracle import prefix_oracle as O
from paper_2608_26574_gb300 import binding as B

pytestmark = pytest.mark.gpu
DEV = "cuda"
U = 2.0 ** -24
TD = {"bf16": torch.bfloat16, "f32": torch.float32}


def _np(t):
    return t.detach().double().cpu().numpy()


def layouts(seqs, seed):
    """Sequences (text, block, after, shadow rows) with random states, confidences and shadow
    sources (any distinct positions of the block, in any order)."""
    rng = np.random.default_rng(seed)
    out = []
    for text, block, after, sh in seqs:
        src = text + rng.permutation(block)[:sh]
        out.append(D.SeqLayout(n_orig=text + block + after, block_start=text,
                               state=rng.integers(0, 3, block).astype(np.uint8),
                               prev_conf=(rng.integers(0, 6, block) / 5).astype(np.float32),
                               shadow_src=src.astype(np.int32)))
    return out


def make(dtype, hq, hkv, d, prefix, seqs, seed=0, spread=1.4):
    lays = layouts(seqs, seed)
    g = torch.Generator(device=DEV).manual_seed(seed + 1)
    rows = sum(x.rows for x in lays)
    rn = lambda *s: torch.randn(*s, generator=g, device=DEV).to(TD[dtype])  # noqa: E731
    t = dict(q=rn(rows, hq, d) * spread, k=rn(rows, hkv, d), v=rn(rows, hkv, d),
             pk=rn(prefix, hkv, d), pv=rn(prefix, hkv, d))
    return lays, t


def meta(lays):
    cat = lambda xs, dt: torch.from_numpy(  # noqa: E731
        np.concatenate([*xs, np.zeros(1)]).astype(dt)).to(DEV)
    return dict(n_orig=[x.n_orig for x in lays], block_start=[x.block_start for x in lays],
                block_len=[x.block_len for x in lays], shadow_len=[x.n_shadow for x in lays],
                state=cat([x.state for x in lays], np.uint8),
                prev_conf=cat([x.prev_conf for x in lays], np.float32),
                shadow_src=cat([x.shadow_src for x in lays], np.int32))


def workspace(t, prefix):
    hq, hkv, d = t["q"].shape[1], t["k"].shape[1], t["q"].shape[2]
    n = B.dard_prefix_attention_workspace_size(t["q"].shape[0], hq, hkv, d, prefix)
    return torch.full((n,), 0x7f, dtype=torch.uint8, device=DEV)  # no preparation needed


def attend(lays, t, ws=True, lse=True, query_start=None, status=None, scale=0.0):
    o = torch.full_like(t["q"], 7.0)
    ls = torch.full(t["q"].shape[:2], 9.0, device=DEV) if lse else None
    call = B.PrefixAttentionCall(**meta(lays), query_start=query_start, status=status, scale=scale,
                                 workspace=workspace(t, t["pk"].shape[0]) if ws else None)
    call(t["q"], t["k"], t["v"], o, t["pk"], t["pv"], lse=ls)
    torch.cuda.synchronize()
    return o, ls


def check_attention(lays, t, o, ls, query_start=None, scale=None):
    want, wlse, mass, dot = O.prefix_attention(*(_np(t[x]) for x in ("q", "k", "v", "pk", "pv")), lays,
                                               query_start, scale)
    d, n = t["q"].shape[2], t["pk"].shape[0] + max(x.rows for x in lays)
    ds = 2 * (d + 4) * U * dot
    rel = 2 * ds + 2.0 ** -20 + 2 * n * U
    got = _np(o)
    none = np.isnan(want).all(-1).all(-1) & np.isnan(wlse).all(-1)
    for lay_none in [none]:
        assert (got[lay_none] == 7.0).all()  # left as they were
    bf16 = t["q"].dtype == torch.bfloat16
    tol = rel[..., None] * mass * 1.01 + (mass * 2.0 ** -7 + np.abs(want) * 2.0 ** -8 * 1.01 if bf16
                                          else np.abs(want) * 4 * U) + 1e-30
    use = ~none
    err = np.abs(got[use] - want[use])
    assert np.isfinite(got[use]).all()
    assert (err <= tol[use]).all(), (err.max(), (err - tol[use]).max())
    if ls is not None:
        gl = _np(ls)
        assert (gl[none] == 9.0).all()
        le = np.abs(gl[use] - wlse[use])
        lt = (ds + 2.0 ** -20 + 2 * n * U + 4 * U * np.abs(wlse))[use]
        assert (le <= lt).all(), (le.max(), (le - lt).max())


CASES = [
    # one token, heads without and with groups, a prefix of every remainder of a tile
    *[("bf16", hq, hkv, d, p, [(1, 0, 0, 0)]) for hq, hkv, d in ((7, 1, 128), (4, 4, 64))
      for p in (0, 1, 63, 64, 65, 127, 128, 129, 700)],
    *[("f32", 6, 2, 64, p, [(1, 0, 0, 0)]) for p in (0, 1, 63, 64, 65, 300)],
    # tiles that span sequences of different kinds, among them one without a block
    ("bf16", 4, 4, 128, 300, [(5, 8, 3, 8), (0, 16, 0, 16), (3, 0, 0, 0), (0, 1, 0, 1), (40, 32, 7, 31)]),
    ("bf16", 14, 2, 64, 130, [(5, 8, 3, 8), (0, 16, 0, 11), (3, 0, 0, 0), (0, 1, 0, 1), (40, 32, 7, 31)]),
    ("f32", 6, 2, 128, 130, [(5, 8, 3, 8), (0, 16, 0, 11), (3, 0, 0, 0), (0, 1, 0, 1), (40, 32, 7, 31)]),
    ("f32", 4, 4, 64, 333, [(0, 32, 0, 32)] * 3),
    # the widest block, own rows past several tiles
    ("bf16", 2, 1, 128, 77, [(200, 128, 90, 128)]),
    ("bf16", 2, 2, 64, 1, [(130, 128, 0, 100), (129, 127, 300, 127)]),
    ("f32", 2, 1, 64, 77, [(200, 128, 90, 128)]),
    # many sequences of one row, and of few
    ("bf16", 8, 2, 128, 513, [(1, 0, 0, 0)] * 200),
    ("bf16", 1, 1, 64, 129, [(2, 3, 1, 3)] * 60),
    ("f32", 3, 3, 64, 65, [(2, 3, 1, 3)] * 60),
    # a group of more heads than a tile has rows
    ("bf16", 150, 1, 64, 200, [(3, 4, 0, 4), (1, 0, 0, 0)]),
    ("f32", 150, 1, 64, 70, [(3, 4, 0, 4), (1, 0, 0, 0)]),
    # more query tiles than the launch's table of sequences holds
    ("bf16", 64, 1, 64, 10, [(14, 9, 3, 9), (1, 0, 0, 0)] * 60),
    ("f32", 64, 1, 64, 10, [(14, 9, 3, 9), (1, 0, 0, 0)] * 60),
    # enough queries for the fp32 kernel's large tiles
    ("f32", 16, 16, 64, 100, [(0, 64, 500, 64)] * 2),
    ("f32", 40, 8, 128, 40, [(0, 32, 300, 32)] * 2),
]


@pytest.mark.parametrize("ws", [True, False])
@pytest.mark.parametrize("dtype,hq,hkv,d,prefix,seqs", CASES)
def test_attention(dtype, hq, hkv, d, prefix, seqs, ws):
    lays, t = make(dtype, hq, hkv, d, prefix, seqs, seed=prefix)
    o, ls = attend(lays, t, ws=ws)
    check_attention(lays, t, o, ls)
    # without lse the same output, and the same bits again
    o2, _ = attend(lays, t, ws=ws, lse=False)
    assert torch.equal(o, o2)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_attention_query_start(dtype):
    """Cached text of a sequence serves as keys only; a sequence without any query."""
    lays, t = make(dtype, 8, 2, 128, 260, [(100, 16, 5, 16), (30, 8, 0, 8), (7, 4, 0, 3), (129, 2, 0, 2)], 3)
    qs = [100, 30 + 8 + 8, 0, 60]
    o, ls = attend(lays, t, query_start=qs)
    check_attention(lays, t, o, ls, query_start=qs)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_attention_equals_step_attention(dtype):
    """The prefix as part of every sequence's own rows: the same sum, by the other kernels."""
    p, d, hq, hkv = 150, 128, 4, 2
    lays, t = make(dtype, hq, hkv, d, p, [(9, 16, 4, 16), (0, 32, 0, 30)], 5)
    o, _ = attend(lays, t)
    parts, n, b0 = {"q": [], "k": [], "v": []}, [], []
    base = 0
    for x in lays:
        for name, pre in (("q", torch.zeros(p, hq, d, device=DEV, dtype=TD[dtype])), ("k", t["pk"]), ("v", t["pv"])):
            parts[name] += [pre, t[name][base:base + x.rows]]
        n.append(p + x.n_orig)
        b0.append(p + x.block_start)
        base += x.rows
    m = meta(lays)
    shift = np.concatenate([np.full(x.n_shadow, p, np.int32) for x in lays] + [np.zeros(1, np.int32)])
    q, k, v = (torch.cat(parts[x]) for x in "qkv")
    full = torch.empty_like(q)
    B.dard_step_attention(q, k, v, full, n, b0, m["block_len"], m["shadow_len"], m["state"], m["prev_conf"],
                          m["shadow_src"] + torch.from_numpy(shift).to(DEV))
    rows, base = [], 0
    for x in lays:
        rows += list(range(base + p, base + p + x.rows))
        base += p + x.rows
    # both within the tolerance of the same sum: twice 1.5 * 2^-7 of the largest value
    lim = 2 * (1.5 * 2 ** -7 if dtype == "bf16" else 1e-5) * float(max(v.abs().max(), 1))
    assert (full[rows].float() - o.float()).abs().max().item() <= lim


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("kind", ["heads first", "slice", "keys and values side by side"])
def test_attention_cache_strides(dtype, kind):
    """Caches in other layouts, inside larger buffers whose other elements are NaN."""
    lays, t = make(dtype, 6, 3, 64, 201, [(3, 8, 0, 8), (0, 5, 2, 5)], 11)
    p, hkv, d = t["pk"].shape
    if kind == "heads first":
        buf = torch.full((2, hkv, p + 50, d), math.nan, device=DEV, dtype=TD[dtype])
        views = [buf[i, :, :p].transpose(0, 1) for i in range(2)]
    elif kind == "slice":
        buf = torch.full((2, p + 9, hkv + 2, d + 64), math.nan, device=DEV, dtype=TD[dtype])
        views = [buf[i, 4:4 + p, 1:1 + hkv, :d] for i in range(2)]
    else:
        buf = torch.full((p + 9, 2, hkv, d), math.nan, device=DEV, dtype=TD[dtype])
        views = [buf[:p, i] for i in range(2)]
    want, _ = attend(lays, t)
    for view, name in zip(views, ("pk", "pv")):
        view.copy_(t[name])
        t[name] = view
    o, ls = attend(lays, t)
    assert torch.equal(o, want)
    check_attention(lays, t, o, ls)


@pytest.mark.parametrize("ws", [True, False])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_attention_hidden_values(dtype, ws):
    """NaN and infinities in keys and values: the rows that see them have them, no other row does."""
    lays, t = make(dtype, 4, 2, 128, 140, [(6, 9, 4, 9), (0, 12, 3, 12), (2, 0, 0, 0), (50, 20, 9, 14)], 21)
    base = np.cumsum([0] + [x.rows for x in lays])
    # values of block positions, of shadow copies, of text; single elements, one sign and both
    t["v"][base[0] + 7, 0, 5] = math.nan
    t["v"][base[0] + lays[0].n_orig + 1, 1, 127] = math.inf
    t["v"][base[1] + 3, 0, 64] = -math.inf
    t["v"][base[1] + lays[1].n_orig + 4, 0, 64] = math.inf
    t["v"][base[1] + 5, 0, 64] = math.inf
    t["v"][base[3] + 55, 1, 0] = math.nan
    o, _ = attend(lays, t, ws=ws)
    want = O.prefix_attention(*(_np(t[x]) for x in ("q", "k", "v", "pk", "pv")), lays)[0]
    got = _np(o)
    assert np.array_equal(np.isnan(got), np.isnan(want))
    assert np.array_equal(np.isinf(got), np.isinf(want))
    assert np.array_equal(np.sign(got[np.isinf(got)]), np.sign(want[np.isinf(want)]))
    fin = np.isfinite(want)
    assert 0 < (~fin).sum() < fin.sum()
    big = np.abs(_np(t["pv"])).max() * 1.2
    assert np.abs(got[fin] - want[fin]).max() <= (1.5 * 2 ** -7 if dtype == "bf16" else 2e-5) * big
    # a key that is NaN: the rows that see it are NaN throughout
    t["v"] = torch.where(torch.isfinite(t["v"]), t["v"], torch.zeros_like(t["v"]))
    t["k"][base[1] + 4, 1, 3] = math.nan
    o, ls = attend(lays, t, ws=ws)
    want, wl = O.prefix_attention(*(_np(t[x]) for x in ("q", "k", "v", "pk", "pv")), lays)[:2]
    assert np.array_equal(np.isnan(_np(o)), np.isnan(want))
    assert np.array_equal(np.isnan(_np(ls)), np.isnan(wl))
    assert np.isnan(want).any() and np.isfinite(want[:base[1]]).all()


@pytest.mark.parametrize("ws", [True, False])
@pytest.mark.parametrize("hq,hkv,d,prefix,seqs", [
    (28, 4, 64, 1900, [(0, 64, 0, 64)] * 3),  # with a workspace in parts
    (28, 4, 64, 1900, [(0, 64, 0, 64)] * 5),
    (48, 2, 128, 700, [(9, 40, 5, 33), (0, 64, 0, 64), (100, 30, 7, 30)]),
    (28, 4, 128, 4097, [(1, 0, 0, 0)]), (1, 1, 64, 20000, [(1, 0, 0, 0)]),  # few queries, many parts
    (28, 4, 128, 1000, [(1, 0, 0, 0)] * 33), (9, 1, 64, 640, [(0, 3, 2, 3)])])
def test_attention_f32_tiles(hq, hkv, d, prefix, seqs, ws):
    """Both fp32 kernels, unsplit and in parts."""
    lays, t = make("f32", hq, hkv, d, prefix, seqs, seed=prefix)
    o, ls = attend(lays, t, ws=ws)
    check_attention(lays, t, o, ls)


def test_attention_hidden_values_f32_tiles():
    """NaN and infinite values of hidden keys in the fp32 kernel for many queries."""
    lays, t = make("f32", 96, 2, 128, 140, [(6, 9, 4, 9), (0, 12, 3, 12), (2, 0, 0, 0), (50, 20, 9, 14)] * 3, 21)
    base = np.cumsum([0] + [x.rows for x in lays])
    t["v"][base[0] + 7, 0, 5] = math.nan
    t["v"][base[1] + 3, 0, 64] = -math.inf
    t["v"][base[1] + 5, 0, 64] = math.inf
    t["v"][base[7] + 55, 1, 0] = math.nan
    o, _ = attend(lays, t)
    want = O.prefix_attention(*(_np(t[x]) for x in ("q", "k", "v", "pk", "pv")), lays)[0]
    got = _np(o)
    assert np.array_equal(np.isnan(got), np.isnan(want))
    assert np.array_equal(np.isinf(got), np.isinf(want))
    fin = np.isfinite(want)
    assert 0 < (~fin).sum() < fin.sum()
    assert np.abs(got[fin] - want[fin]).max() <= 2e-5 * np.abs(_np(t["pv"])).max() * 1.2


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_attention_extreme_scores(dtype):
    """Scores far apart: one key takes all the weight, and its value comes back exactly."""
    lays, t = make(dtype, 2, 2, 64, 300, [(1, 0, 0, 0), (0, 4, 0, 4)], 8)
    t["q"].zero_()
    t["q"][..., 0] = 30.0
    t["pk"][..., 0] = -30.0
    t["k"][..., 0] = -30.0
    t["pk"][211, :, 0] = 60.0
    o, ls = attend(lays, t)
    assert torch.equal(o, t["pv"][211][None].expand_as(o))
    assert np.allclose(_np(ls), 30 * 60 / 8.0, rtol=1e-6)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_attention_marks(dtype):
    """A bad state byte, a repeated and a stray shadow source: status bits, fallback, rows unwritten."""
    lays, t = make(dtype, 2, 1, 64, 70, [(4, 8, 2, 4)], 9)
    m = meta(lays)
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    m["state"][2] = 9
    src = np.array([5, 7, 5, 40], np.int32)
    m["shadow_src"] = torch.from_numpy(src).to(DEV)
    o = torch.full_like(t["q"], 7.0)
    ls = torch.full(t["q"].shape[:2], 9.0, device=DEV)
    B.PrefixAttentionCall(**m, status=status, workspace=workspace(t, 70))(
        t["q"], t["k"], t["v"], o, t["pk"], t["pv"], lse=ls)
    torch.cuda.synchronize()
    assert status.item() == B.STATUS_BAD_STATE | B.STATUS_BAD_SHADOW
    n = lays[0].n_orig
    assert (o[n + 2:] == 7.0).all() and (ls[n + 2:] == 9.0).all()
    # the oracle without the rows that count for nothing, the bad state read as M
    st = lays[0].state.copy()
    st[2] = 0
    lay = D.SeqLayout(n, 4, st, lays[0].prev_conf, src[:2])
    keep = {x: t[x][:n + 2] for x in ("q", "k", "v")}
    check_attention([lay], {**t, **keep}, o[:n + 2], ls[:n + 2])


def test_attention_scale_and_nothing_to_do():
    lays, t = make("bf16", 4, 2, 64, 90, [(3, 8, 0, 8)], 2)
    o, ls = attend(lays, t, scale=0.31)
    check_attention(lays, t, o, ls, scale=float(np.float32(0.31)))
    o, ls = attend(lays, t, query_start=[lays[0].rows])  # no query rows
    assert (o == 7.0).all() and (ls == 9.0).all()


def test_attention_rows_behind_the_last_sequence():
    lays, t = make("bf16", 4, 4, 64, 90, [(3, 8, 0, 8)], 2)
    pad = {x: torch.cat([t[x], torch.full((5, *t[x].shape[1:]), math.nan, device=DEV, dtype=t[x].dtype)])
           for x in ("q", "k", "v")}
    o, ls = attend(lays, {**t, **pad})
    n = t["q"].shape[0]
    assert (o[n:] == 7.0).all() and (ls[n:] == 9.0).all()
    check_attention(lays, t, o[:n], ls[:n])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_attention_graphs_and_streams(dtype):
    """A captured call replayed on new data, and two graphs that share a workspace in one stream."""
    lays, t = make(dtype, 8, 1, 128, 900, [(0, 6, 0, 6)], 4)
    o, ls = torch.zeros_like(t["q"]), torch.zeros(t["q"].shape[:2], device=DEV)
    ws = workspace(t, 900)
    call = B.PrefixAttentionCall(**meta(lays), workspace=ws)
    lays2, t2 = make(dtype, 4, 4, 128, 400, [(2, 3, 0, 3)] * 2, 6)
    o2 = torch.zeros_like(t2["q"])
    call2 = B.PrefixAttentionCall(**meta(lays2), workspace=ws)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        call(t["q"], t["k"], t["v"], o, t["pk"], t["pv"], lse=ls)
        call2(t2["q"], t2["k"], t2["v"], o2, t2["pk"], t2["pv"])
        s.synchronize()
        g1, g2 = torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()
        with torch.cuda.graph(g1, stream=s):
            call(t["q"], t["k"], t["v"], o, t["pk"], t["pv"], lse=ls)
        with torch.cuda.graph(g2, stream=s):
            call2(t2["q"], t2["k"], t2["v"], o2, t2["pk"], t2["pv"])
        t["pk"].mul_(-1)
        t2["q"].mul_(0.5)
        for _ in range(3):
            g1.replay()
            g2.replay()
        s.synchronize()
    want, wl = attend(lays, t)
    assert torch.equal(o, want) and torch.equal(ls, wl)
    assert torch.equal(o2, attend(lays2, t2)[0])


def test_attention_long_cache_offsets():
    """A cache whose elements pass 2^32: rows behind that border count like the others."""
    p, hkv, d = (1 << 20) + 77, 32, 128
    g = torch.Generator(device=DEV).manual_seed(0)
    pk = torch.zeros(p, hkv, d, device=DEV, dtype=torch.bfloat16)
    pv = torch.zeros(p, hkv, d, device=DEV, dtype=torch.bfloat16)
    lays, t = make("bf16", 32, hkv, d, 0, [(0, 2, 0, 2)], 1)
    # all scores are 0 but those of the last keys
    last = torch.randn(64, hkv, d, generator=g, device=DEV) * 4
    pk[-64:] = last.to(torch.bfloat16)
    pv[-64:] = torch.randn(64, hkv, d, generator=g, device=DEV).to(torch.bfloat16)
    t.update(pk=pk, pv=pv)
    t["k"].zero_()
    t["v"].zero_()
    o, ls = attend(lays, t)
    q = t["q"].double()
    z = torch.einsum("rhd,khd->rhk", q, pk[-64:].double()) / math.sqrt(d)
    total = torch.exp(z).sum(-1) + (p - 64 + lays[0].n_orig)
    want = torch.einsum("rhk,khd->rhd", torch.exp(z), pv[-64:].double()) / total[..., None]
    mass = torch.einsum("rhk,khd->rhd", torch.exp(z), pv[-64:].double().abs()) / total[..., None]
    # 2^13 key tiles of weight-one additions in fp32: 2^-11 relative at most
    assert ((o.double() - want).abs() <= mass * (2.0 ** -7 + 2.0 ** -8 + 2.0 ** -11) + 1e-9).all()
    assert ((ls.double() - torch.log(total)).abs() <= 2.0 ** -11).all()


# ------------------------------------------------------------------------------ weights
def weigh(q, lse, pk, w_in=None, decay=1.0, ws=True, scale=0.0, out=None):
    rows, hq, d = q.shape
    p, hkv = pk.shape[:2]
    n = B.dard_prefix_weights_workspace_size(rows, hq, hkv, d, p)
    w = torch.full((hkv, p), math.nan, device=DEV) if out is None else out
    B.PrefixWeightsCall(scale, decay, torch.full((n,), 0x7f, dtype=torch.uint8, device=DEV) if ws else None)(
        q, lse, pk, w, weights_in=w_in)
    torch.cuda.synchronize()
    return w


def check_weights(q, lse, pk, got, w_in=None, decay=1.0, scale=None):
    want, new, dot = O.prefix_weights(_np(q), _np(lse), _np(pk), None if w_in is None else _np(w_in), decay, scale)
    d, terms = q.shape[2], q.shape[0] * q.shape[1] // pk.shape[1]
    fin = np.abs(_np(lse))
    big = fin[np.isfinite(fin)].max(initial=0.0)
    rel = 2 * (d + 4) * U * dot + 2.0 ** -20 + 4 * U * big + (64 + terms / 64) * 2 * U
    tol = rel * new + 4 * U * np.abs(want) + 1e-37
    err = np.abs(_np(got) - want)
    assert (err <= tol).all(), (err.max(), (err - tol).max())


W_CASES = [("bf16", 7, 1, 128, 1, 1), ("bf16", 28, 4, 128, 1, 700), ("bf16", 4, 4, 64, 5, 129),
           ("bf16", 28, 4, 64, 37, 300), ("bf16", 32, 32, 128, 130, 127), ("bf16", 150, 1, 64, 9, 257),
           ("bf16", 2, 2, 128, 3000, 65), ("bf16", 96, 1, 64, 700, 128), ("f32", 6, 2, 64, 1, 1),
           ("f32", 6, 2, 64, 77, 1023), ("f32", 28, 4, 128, 40, 130), ("f32", 1, 1, 64, 3000, 64),
           ("f32", 150, 1, 128, 3, 200)]


@pytest.mark.parametrize("ws", [True, False])
@pytest.mark.parametrize("dtype,hq,hkv,d,rows,prefix", W_CASES)
def test_weights(dtype, hq, hkv, d, rows, prefix, ws):
    _, t = make(dtype, hq, hkv, d, prefix, [(rows, 0, 0, 0)], rows)
    lse = torch.randn(rows, hq, device=DEV, generator=torch.Generator(DEV).manual_seed(1)) + 7
    lse[rows // 2] = math.inf  # a row that is no query, whatever its q holds
    q = t["q"]
    bad = q.clone()
    bad[rows // 2] = math.nan
    got = weigh(bad, lse, t["pk"], ws=ws)
    check_weights(q, lse, t["pk"], got)
    assert torch.equal(got, weigh(q, lse, t["pk"], ws=ws))  # equal bits, NaN or not
    # a decayed earlier sum, in another buffer, in place, and in rows of a wider one
    w_in = torch.rand(hkv, prefix, device=DEV) * 3
    out = weigh(bad, lse, t["pk"], w_in, 0.75, ws)
    check_weights(q, lse, t["pk"], out, w_in, 0.75)
    wide = torch.full((hkv, prefix + 5), 5.0, device=DEV)
    wide[:, 2:2 + prefix] = w_in
    weigh(bad, lse, t["pk"], wide[:, 2:2 + prefix], 0.75, ws, out=wide[:, 2:2 + prefix])
    assert torch.equal(wide[:, 2:2 + prefix], out)
    assert (wide[:, :2] == 5).all() and (wide[:, 2 + prefix:] == 5).all()


def test_weights_all_rows_off_and_no_rows():
    _, t = make("bf16", 8, 2, 64, 200, [(9, 0, 0, 0)], 1)
    lse = torch.full((9, 8), math.inf, device=DEV)
    assert (weigh(t["q"], lse, t["pk"]) == 0).all()
    w = torch.rand(2, 200, device=DEV)
    assert torch.equal(weigh(t["q"][:0], lse[:0], t["pk"], w, 0.5), w * 0.5)
    assert (weigh(t["q"][:0], lse[:0], t["pk"]) == 0).all()


@pytest.mark.parametrize("ws", [True, False])
@pytest.mark.parametrize("d,hq,hkv,rows,prefix", [(64, 4, 2, 40, 200), (128, 6, 2, 77, 300), (128, 1, 1, 1, 1),
                                                  (128, 130, 1, 3, 129), (64, 3, 3, 200, 64)])
def test_weights_of_large_scores(d, hq, hkv, rows, prefix, ws):
    """Scores of 512 beside 1e-4 per element, far above their lse: an fp32 sum of them that is cut or
    rounded element by element is off by up to a unit of 6e-5 each time, times 1 / sqrt(d) the relative
    error of the weight (6e-5 to 9e-5 here without exact scores). They leave the rounding of the exponent (below 32 in base 2:
    32 * 2^-24 * ln 2 = 1.4e-6), of the exponential (2^-22) and of the sums (16 * 2^-24)."""
    g = torch.Generator(device=DEV).manual_seed(d + rows)

    def make_rows(n, h):
        x = 1 + torch.randint(0, 128, (n, h, d), generator=g, device=DEV) / 128  # 8 bits
        x *= 2.0 ** -7
        x[..., :8] = 8.0
        return x.to(torch.bfloat16)
    q, pk = make_rows(rows, hq), make_rows(prefix, hkv)
    lse = 512 / d ** 0.5 - 10 - torch.rand(rows, hq, generator=g, device=DEV)
    got = weigh(q, lse, pk, None, 0.5, ws)
    want = O.prefix_weights(_np(q), _np(lse), _np(pk))[0]
    assert want.min() > 2e4
    rel = np.abs(_np(got) - want) / want
    assert rel.max() <= 32 * U * math.log(2) + 2.0 ** -22 + 16 * U, rel.max()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_weights_strides(dtype):
    _, t = make(dtype, 6, 3, 64, 201, [(30, 0, 0, 0)], 11)
    lse = torch.full((30, 6), 5.0, device=DEV)
    buf = torch.full((3, 260, 64), math.nan, device=DEV, dtype=TD[dtype])
    view = buf[:, :201].transpose(0, 1)
    view.copy_(t["pk"])
    assert torch.equal(weigh(t["q"], lse, view), weigh(t["q"], lse, t["pk"]))


# ------------------------------------------------------------------------------ eviction
def evict(w, k, v, keep, first=0, last=0):
    hkv, d = k.shape[1:]
    kept = torch.full((hkv, keep), -5, dtype=torch.int32, device=DEV)
    ko, vo = (torch.full((keep, hkv, d), 3.0, dtype=k.dtype, device=DEV) for _ in range(2))
    wo = torch.full((hkv, keep), -1.0, device=DEV)
    B.dard_prefix_evict(w, k, v, kept, ko, vo, wo, keep_first=first, keep_last=last)
    torch.cuda.synchronize()
    return kept, ko, vo, wo


def check_evict(w, k, v, keep, first=0, last=0):
    kept, ko, vo, wo = evict(w, k, v, keep, first, last)
    want = O.prefix_evict(_np(w), keep, first, last)
    assert np.array_equal(kept.cpu().numpy(), want)
    at = torch.from_numpy(want).long().to(DEV)
    heads = torch.arange(k.shape[1], device=DEV)[:, None]
    for got, src in ((ko, k), (vo, v)):
        assert torch.equal(got.view(torch.uint8), src[at, heads].transpose(0, 1).contiguous().view(torch.uint8))
    assert torch.equal(wo.view(torch.int32), w.gather(1, at).view(torch.int32))


E_CASES = [(1, 1, 0, 0), (1, 1, 1, 0), (2, 1, 0, 1), (33, 5, 2, 3), (100, 100, 0, 0), (704, 512, 4, 64),
           (4099, 1111, 1, 33), (8193, 8000, 0, 0), (20000, 1, 0, 0), (40000, 20001, 7, 500), (5, 0, 0, 0)]


@pytest.mark.parametrize("kind", ["random", "ties", "equal", "special"])
@pytest.mark.parametrize("prefix,keep,first,last", E_CASES)
def test_evict(prefix, keep, first, last, kind):
    g = torch.Generator(DEV).manual_seed(prefix)
    hkv, d = 3, 64
    w = torch.exp(2 * torch.randn(hkv, prefix, generator=g, device=DEV))
    if kind == "ties":
        w = torch.randint(0, 4, (hkv, prefix), generator=g, device=DEV).float()
    elif kind == "equal":
        w = torch.full((hkv, prefix), 0.25, device=DEV)
    elif kind == "special":
        pool = torch.tensor([math.nan, -math.nan, math.inf, -math.inf, 0.0, -0.0, 1e-45, -1e-45, 1.0, -3.0, 3.4e38],
                            device=DEV)
        w = pool[torch.randint(0, len(pool), (hkv, prefix), generator=g, device=DEV)]
    dt = torch.bfloat16 if prefix % 2 else torch.float32
    k, v = (torch.randn(prefix, hkv, d, generator=g, device=DEV).to(dt) for _ in range(2))
    check_evict(w, k, v, keep, first, last)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_evict_strides(dtype):
    """Weights in a wider buffer, caches with the heads first, outputs inside a larger cache."""
    hkv, p, d, keep = 5, 300, 128, 77
    w = torch.rand(hkv, p + 3, device=DEV)[:, 1:1 + p]
    k, v = (torch.randn(hkv, p + 2, d, device=DEV).to(TD[dtype])[:, :p].transpose(0, 1) for _ in range(2))
    out = torch.full((2, keep + 4, hkv, d + 64), 3.0, device=DEV, dtype=TD[dtype])
    kept = torch.empty(hkv, keep, dtype=torch.int32, device=DEV)
    B.dard_prefix_evict(w, k, v, kept, out[0, :keep, :, :d], out[1, :keep, :, :d], keep_last=9)
    torch.cuda.synchronize()
    want = O.prefix_evict(_np(w), keep, 0, 9)
    assert np.array_equal(kept.cpu().numpy(), want)
    at, heads = torch.from_numpy(want).long().to(DEV), torch.arange(hkv, device=DEV)[:, None]
    for i, src in enumerate((k, v)):
        assert torch.equal(out[i, :keep, :, :d], src[at, heads].transpose(0, 1))
        assert (out[i, keep:] == 3).all() and (out[i, :, :, d:] == 3).all()


def test_evict_long():
    """More candidates than one CTA takes at a time, and indices behind 2^20."""
    p, keep = (1 << 20) + 13, 4097
    g = torch.Generator(DEV).manual_seed(1)
    w = torch.rand(2, p, generator=g, device=DEV)
    k, v = (torch.randn(p, 2, 64, generator=g, device=DEV).to(torch.bfloat16) for _ in range(2))
    kept, ko, vo, wo = evict(w, k, v, keep, 3, 100)
    mid = torch.sort(w[:, 3:p - 100], dim=1, descending=True, stable=True).indices[:, :keep - 103]
    ends = [torch.arange(3, device=DEV).expand(2, -1), torch.arange(p - 100, p, device=DEV).expand(2, -1)]
    want = torch.cat([ends[0], mid.sort(1).values + 3, ends[1]], 1)
    assert torch.equal(kept.long(), want)
    assert torch.equal(ko, k[want, torch.arange(2, device=DEV)[:, None]].transpose(0, 1))
    assert torch.equal(vo, v[want, torch.arange(2, device=DEV)[:, None]].transpose(0, 1))
    assert torch.equal(wo, w.gather(1, want))


# ------------------------------------------------------------------------------ together
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_cache_in_use(dtype):
    """Attention, the weights it spent, eviction by them, attention over what is left: as one run,
    captured and replayed, against the oracle throughout."""
    hq, hkv, d, p, keep = 8, 2, 64, 391, 150
    lays, t = make(dtype, hq, hkv, d, p, [(4, 16, 0, 16), (0, 9, 2, 9), (30, 4, 0, 4)], 13)
    qs = [0, 0, 30]
    rows = t["q"].shape[0]
    o, o2 = torch.zeros_like(t["q"]), torch.zeros_like(t["q"])
    lse = torch.full((rows, hq), math.inf, device=DEV)
    lse2 = lse.clone()
    w, kept = torch.zeros(hkv, p, device=DEV), torch.zeros(hkv, keep, dtype=torch.int32, device=DEV)
    k2, v2 = (torch.zeros(keep, hkv, d, dtype=TD[dtype], device=DEV) for _ in range(2))
    w2 = torch.zeros(hkv, keep, device=DEV)
    ws = torch.empty(max(B.dard_prefix_attention_workspace_size(rows, hq, hkv, d, p),
                         B.dard_prefix_weights_workspace_size(rows, hq, hkv, d, p)),
                     dtype=torch.uint8, device=DEV)
    attention = B.PrefixAttentionCall(**meta(lays), query_start=qs, workspace=ws)
    weights, drop = B.PrefixWeightsCall(workspace=ws), B.PrefixEvictCall(2, 20)

    def run():
        attention(t["q"], t["k"], t["v"], o, t["pk"], t["pv"], lse=lse)
        weights(t["q"], lse, t["pk"], w, weights_in=w)
        drop(w, t["pk"], t["pv"], kept, k2, v2, w2)
        attention(t["q"], t["k"], t["v"], o2, k2, v2, lse=lse2)

    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        run()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            run()
        w.zero_()
        graph.replay()
        s.synchronize()
    first = torch.isinf(lse).all(1)
    assert first.sum().item() == 30  # the rows that are no queries
    got = {**t}
    o_want, l_want = O.prefix_attention(*(_np(t[x]) for x in ("q", "k", "v", "pk", "pv")), lays, qs)[:2]
    use = ~np.isnan(l_want).all(1)
    assert np.abs(_np(lse)[use] - l_want[use]).max() < 1e-4
    check_weights(t["q"], lse, t["pk"], w)
    # every query's weights over the prefix and its own keys add up to 1
    assert np.array_equal(kept.cpu().numpy(), O.prefix_evict(_np(w), keep, 2, 20))
    got.update(pk=k2, pv=v2)
    o2[first] = 7.0
    lse2[first] = 9.0
    check_attention(lays, got, o2, lse2, query_start=qs)
