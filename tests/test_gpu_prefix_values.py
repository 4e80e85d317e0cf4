"""The shared prefix's operators where sums of many parts, values that are not finite and roundings
meet, against the float64 oracle (helpers and tolerances as in test_gpu_prefix.py)."""
import math

import numpy as np
import pytest
import torch

from oracle import prefix_oracle as O

from . import test_gpu_prefix as T

pytestmark = pytest.mark.gpu
DEV = "cuda"
U = T.U


def _same_nan(lays, t, ws):
    o, ls = T.attend(lays, t, ws=ws)
    want, wl = O.prefix_attention(*(T._np(t[x]) for x in ("q", "k", "v", "pk", "pv")), lays)[:2]
    assert np.array_equal(np.isnan(T._np(o)), np.isnan(want))
    assert np.array_equal(np.isnan(T._np(ls)), np.isnan(wl))
    fin = np.isfinite(wl)
    assert np.abs(T._np(ls)[fin] - wl[fin]).max(initial=0.0) <= 1e-4
    return want


PART_CASES = [("bf16", 28, 4, 128, 4096, [(1, 0, 0, 0)]), ("f32", 28, 4, 128, 4096, [(1, 0, 0, 0)]),
              ("bf16", 28, 4, 64, 2000, [(0, 5, 0, 5)] * 2), ("f32", 28, 4, 64, 1900, [(0, 64, 0, 64)] * 3)]


@pytest.mark.parametrize("ws", [True, False])
@pytest.mark.parametrize("dtype,hq,hkv,d,prefix,seqs", PART_CASES)
@pytest.mark.parametrize("first,n", [(0, 128), (0, 1024), (256, 64), (1024, 512), (1800, 2200), (0, 5000)])
def test_attention_nan_throughout_a_part(dtype, hq, hkv, d, prefix, seqs, first, n, ws):
    """Runs of NaN keys that fill whole parts of a split (one, a quarter of them, all): every row sees
    them, so that its output and its normaliser are NaN, in parts or not."""
    lays, t = T.make(dtype, hq, hkv, d, prefix, seqs, 5)
    t["pk"][first:first + n, 1, 3] = math.nan
    want = _same_nan(lays, t, ws)
    assert np.isnan(want[:, hq // hkv:2 * hq // hkv]).all() and np.isfinite(want[:, :hq // hkv]).all()


@pytest.mark.parametrize("ws", [True, False])
@pytest.mark.parametrize("dtype,hq,hkv,d,prefix,seqs", PART_CASES)
def test_attention_nan_in_the_last_part(dtype, hq, hkv, d, prefix, seqs, ws):
    """A row whose own keys alone are NaN (the last part of a split may hold nothing else)."""
    lays, t = T.make(dtype, hq, hkv, d, prefix, seqs, 5)
    t["k"][:lays[0].rows, 2] = math.nan
    want = _same_nan(lays, t, ws)
    assert np.isnan(want).any() and np.isfinite(want).any()


@pytest.mark.parametrize("ws", [True, False])
@pytest.mark.parametrize("dtype,hq,hkv,d,prefix,seqs", PART_CASES)
def test_attention_nan_query_and_parts_without_weight(dtype, hq, hkv, d, prefix, seqs, ws):
    """A NaN query head: NaN, its normaliser too. Keys whose scores are -inf over whole parts have no
    weight, and the other keys' sum is left as it is; a NaN value behind one of them is seen all the same."""
    lays, t = T.make(dtype, hq, hkv, d, prefix, seqs, 5)
    t["q"][..., 3] = t["q"][..., 3].abs() + 0.5
    t["pk"][:1200, :, 3] = -math.inf
    t["pv"][100, 3, 5] = math.nan
    t["q"][0, 2, 7] = math.nan
    want = _same_nan(lays, t, ws)
    assert np.isnan(want[0, 2]).all() and np.isfinite(want[0, 3]).all() and np.isnan(want[:, -1, 5]).all()


@pytest.mark.parametrize("ws", [True, False])
@pytest.mark.parametrize("seqs,prefix", [([(1, 0, 0, 0)] * 12, 201), ([(0, 6, 0, 6)] * 3, 130), ([(1, 0, 0, 0)], 4500)])
@pytest.mark.parametrize("d", [64, 128])
def test_attention_of_equal_values(d, seqs, prefix, ws):
    """Weights that all round the same way (one key ahead, the others alike behind it, at every distance):
    an output that adds rounded weights is divided by their sum, so that equal values come back as they
    are. (The sum of the unrounded ones is off by up to 2^-8, half a step of these values by 2^-9.)"""
    lays, t = T.make("bf16", 4, 2, d, prefix, seqs, 3)
    rows = t["q"].shape[0]
    for x in ("q", "k", "pk"):
        t[x].zero_()
    # q.k = 0 for the first key of the prefix and -x for all others, x a different one for each query
    x = torch.linspace(0.1, 2.0, rows * 4, device=DEV).view(rows, 4)
    t["q"][..., 0] = x.to(torch.bfloat16)
    t["k"][..., 0] = t["pk"][..., 0] = -d ** 0.5
    t["pk"][0] = 0
    for x in ("v", "pv"):
        t[x].fill_(1.9921875)  # the relative half step is smallest just below 2
    o, ls = T.attend(lays, t, ws=ws)
    assert (o == 1.9921875).all(), o[o != 1.9921875]
    T.check_attention(lays, t, o, ls)


@pytest.mark.parametrize("hq,hkv,rows", [(7, 1, 40), (8, 1, 40), (14, 2, 1), (16, 2, 3), (150, 1, 9), (3, 3, 130),
                                         (9, 3, 43)])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("ws", [True, False])
def test_weights_of_keys_that_are_not_finite(dtype, hq, hkv, rows, ws):
    """Infinite elements make a key's scores +inf or -inf: its weight is +inf or what the other rows give
    it. A NaN makes it NaN, but where no row counts (lse = +inf) everything is 0. Whatever number of query
    heads a tile has room for."""
    _, t = T.make(dtype, hq, hkv, 64, 300, [(rows, 0, 0, 0)], 5)
    q, pk = t["q"], t["pk"]
    q[..., 3] = q[..., 3].abs() + 0.25
    lse = torch.rand(rows, hq, device=DEV, generator=torch.Generator(DEV).manual_seed(2)) + 7
    lse[rows // 2, hq // 2] = math.inf
    clean = pk.clone()
    pk[5, :, 3] = math.inf
    pk[6, :, 3] = -math.inf
    pk[200, 0, 3] = -math.inf
    pk[7, hkv - 1, 9] = math.nan
    got = T.weigh(q, lse, pk, ws=ws)
    inf = torch.zeros(hkv, 300, dtype=torch.bool, device=DEV)
    inf[:, 5] = True
    none, nan = torch.zeros_like(inf), torch.zeros_like(inf)
    none[:, 6] = none[0, 200] = nan[hkv - 1, 7] = True
    if (rows, hq // hkv) == (1, 1):
        inf[:, 5] = lse[0, 0] != math.inf
    assert torch.equal(got == math.inf, inf)
    assert torch.equal(torch.isnan(got), nan)
    assert (got[none] == 0).all()
    odd = inf | none | nan
    want = T.weigh(q, lse, clean, ws=ws)
    assert torch.equal(got[~odd], want[~odd])
    assert (T.weigh(q, torch.full_like(lse, math.inf), pk, ws=ws) == 0).all()


@pytest.mark.parametrize("ws", [True, False])
@pytest.mark.parametrize("scale", [0.25, 0.0])
def test_weights_of_exact_scores(scale, ws):
    """Scores of a few large products, which no sum cuts or rounds, next to their normalisers: z = 512 scale,
    up to 128. The normaliser enters as a 32-bit number in base 2, which is taken into account here (values
    whose product lies halfway between two of them are left out); what remains is the exponent itself (below 8
    in base 2: 4 u ln 2), the exponential (2^-22), 16 additions and the scale's rounding, which counts for the
    difference of at most 5. (A normaliser off by 4e-8 of itself is 5e-6 of the weight.)"""
    d, hq, rows, prefix = 128, 8, 64, 300
    q, pk = (torch.zeros(n, h, d, dtype=torch.bfloat16, device=DEV) for n, h in ((rows, hq), (prefix, 1)))
    q[..., 16:24] = pk[..., 16:24] = 8.0
    c = scale or d ** -0.5
    z = 512 * c
    unit = float(np.float32(np.float32(c) * np.float32(math.log2(math.e)))) / c
    cand = (z + 2 + np.random.default_rng(1).random(4000) * 3).astype(np.float32)
    prod = cand.astype(np.float64) * unit
    near = prod.astype(np.float32).astype(np.float64)
    use = np.abs(prod - near) < 0.48 * np.spacing(near.astype(np.float32))
    cand, near = cand[use][:rows * hq], near[use][:rows * hq]
    got = T.weigh(q, torch.from_numpy(cand).to(DEV).view(rows, hq), pk, ws=ws, scale=scale)
    want = np.exp2(z * unit - near).sum()
    assert want / (rows * hq) * 32 < 4  # far from the sums that are formed another way
    tol = 4 * U * math.log(2) + 2.0 ** -22 + 16 * U
    rel = np.abs(T._np(got) / want - 1).max()
    assert rel <= tol, (rel, tol)


@pytest.mark.parametrize("ws", [True, False])
@pytest.mark.parametrize("prefix", [1, 2, 5])
@pytest.mark.parametrize("d,hq,hkv,rows", [(128, 8, 2, 128), (64, 6, 2, 77)])
def test_weights_of_large_scores_behind_few_keys(d, hq, hkv, rows, prefix, ws):
    """The scores of test_weights_of_large_scores behind a prefix of a few keys, each with its share of
    every query's weight: their sums are exact too (6e-5 off if they are formed on the tensor cores, each
    element a unit of a running sum of 512). Left are the exponent's rounding (below 4 in base 2: 4 u ln 2), the
    exponential's (2^-22) and at most 24 additions; and 32 columns of a tile that hold so few queries that
    their sum stays below 8, whose terms keep the cut: at most a unit of 512 (2^-14) for each of d - 8 elements."""
    g = torch.Generator(device=DEV).manual_seed(d + rows)

    def make_rows(n, h):
        x = 1 + torch.randint(0, 128, (n, h, d), generator=g, device=DEV) / 128  # 8 bits
        x *= 2.0 ** -7
        x[..., :8] = 8.0
        return x.to(torch.bfloat16)
    q, pk = make_rows(rows, hq), make_rows(prefix, hkv)
    z = torch.einsum("rhgd,khd->rhgk", q.double().view(rows, hkv, -1, d), pk.double()) / d ** 0.5
    share = min(prefix, 3)  # a key's part: above a quarter
    lse = (z.mean(-1) + math.log(share)).float().view(rows, hq)
    got = T.weigh(q, lse, pk, ws=ws)
    want = O.prefix_weights(T._np(q), T._np(lse), T._np(pk))[0]
    rel = np.abs(T._np(got) - want) / want
    group, per_tile = hq // hkv, 128 // (hq // hkv)
    tiles = [min(per_tile, rows - r) * group for r in range(0, rows, per_tile)]
    words = [min(32, n - c) for n in tiles for c in range(0, n, 32)]
    cut = sum(n for n in words if n / share <= 8) / (rows * group) * (d - 8) * 2.0 ** -14 / d ** 0.5
    assert rel.max() <= 4 * U * math.log(2) + 2.0 ** -22 + 24 * U + cut, (rel.max(), cut)


@pytest.mark.parametrize("x", [0.7, 1.1, 2.3])
def test_weights_f32_of_many_equal_terms(x):
    """73728 equal terms for each key, in one run (no workspace): every addition to a running sum would round the
    same way (up to 2^-24 of the sum each time, 6e-5 in all). The kernel keeps what the roundings of its
    long sums cut off, which leaves a tile's 4 terms of a thread, the 16 threads' sums and the last
    roundings (12 u), the term's own error (the exponential 2^-22, its exponent 8 u ln 2)."""
    rows, hq, d, prefix = 9216, 8, 64, 130
    g = torch.Generator(device=DEV).manual_seed(1)
    q = torch.randn(1, 1, d, device=DEV, generator=g).expand(rows, hq, d).contiguous()
    pk = torch.randn(prefix, 1, d, device=DEV, generator=g) * 0.1
    lse = torch.full((rows, hq), x, device=DEV)
    got = T.weigh(q, lse, pk, ws=False)
    want, _, dot = O.prefix_weights(T._np(q[:1, :1]), T._np(lse[:1, :1]), T._np(pk))
    want = want * (rows * hq)
    rel = np.abs(T._np(got) - want) / want
    tol = 2 * (d + 4) * U * dot + 2.0 ** -22 + 8 * U * math.log(2) + 4 * U * x + 12 * U
    assert (rel <= tol).all(), (rel.max(), (rel - tol).max())
