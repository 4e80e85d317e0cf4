"""Pins of the experts' MLP oracle: closed forms, brute force and torch's own conversions, on
the CPU. Nothing here calls the library."""
import itertools
import math

import numpy as np
import pytest
import torch

from oracle import mlp_oracle as O


def _e4m3_values():
    """Every finite e4m3 value, from torch's table of the type."""
    codes = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    return np.unique(codes[np.isfinite(codes)])


def test_e4m3_keeps_every_value_and_picks_the_nearest():
    v = _e4m3_values()
    assert v.max() == O.E4M3_MAX and np.array_equal(O.e4m3(v), v)
    rng = np.random.default_rng(0)
    x = np.concatenate([rng.uniform(-448, 448, 500), rng.normal(0, 0.02, 500)])
    near = v[np.abs(x[:, None] - v[None]).argmin(1)]
    assert np.array_equal(O.e4m3(x), near)
    # ties between neighbours go to the even code: the same as torch's conversion
    mid = (v[1:] + v[:-1]) / 2
    want = torch.from_numpy(mid).float().to(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(O.e4m3(mid), want)


def test_round_bf16_is_torchs():
    rng = np.random.default_rng(1)
    x = rng.normal(size=4000) * 10.0 ** rng.integers(-30, 30, 4000)
    x = np.concatenate([x, [0.0, np.inf, -np.inf, 1e-40]]).astype(np.float32)
    want = torch.from_numpy(x).to(torch.bfloat16).double().numpy()
    assert np.array_equal(O.round_bf16(x), want)


@pytest.mark.parametrize("top,byte", [
    (448.0, 127), (448.0000001, 128), (447.9, 127), (224.0, 126), (225.0, 127), (1.75, 119),
    (1.7500001, 120), (0.0, 0), (2.0 ** -149, 0), (448 * 2.0 ** -127, 0), (3.4e38, 247)])
def test_scale_byte_closed_forms(top, byte):
    v = np.zeros(32)
    v[5] = -top
    codes, b = O.mx_round(v)
    assert b == byte and np.abs(codes).max() <= O.E4M3_MAX


def test_scale_is_the_smallest():
    rng = np.random.default_rng(2)
    v = rng.normal(size=(200, 64)) * 2.0 ** rng.integers(-20, 20, (200, 1))
    _, b = O.mx_round(v)
    top = np.abs(v).reshape(200, 2, 32).max(-1)
    e = b.astype(int) - 127
    assert (top <= 448 * 2.0 ** e).all() and (top > 448 * 2.0 ** (e - 1)).all()


@pytest.mark.parametrize("bad", [np.nan, np.inf, -np.inf])
def test_bad_values_spoil_their_block_only(bad):
    v = np.ones((1, 96))
    v[0, 40] = bad
    codes, b = O.mx_round(v)
    assert b[0].tolist() == [119, 255, 119]  # 2^-8: 1 becomes 256
    assert np.isnan(codes[0, 32:64]).all() and (codes[0, :32] == 256).all() and \
        (codes[0, 64:] == 256).all()


def test_tiles_place_every_scale_once():
    s = np.arange(1, 131 * 5 + 1).reshape(131, 5) % 251 + 1
    t = O.tile_scales(s.astype(np.uint8))
    assert t.shape == (2, 2, 512) and np.count_nonzero(t) == 131 * 5
    assert t[0, 0, 0] == s[0, 0] and t[0, 0, 16] == s[1, 0] and t[0, 0, 4] == s[32, 0]
    assert t[0, 0, 3] == s[0, 3] and t[0, 1, 0] == s[0, 4] and t[1, 0, 2 * 16 + 1] == s[130, 1]


def test_norm_closed_forms():
    x = np.array([[3.0, -4.0, 0.0, 0.0]])
    r, n = O.residual_norm(x, None, None, 0.0, False)
    assert np.allclose(n, x / 2.5, rtol=1e-15) and np.array_equal(r, x)
    r, n = O.residual_norm(x, x, np.array([1.0, 2.0, 1.0, 1.0]), 0.0, True)
    assert np.array_equal(r, 2 * x) and np.allclose(n, x / 2.5 * [1, 2, 1, 1], rtol=1e-15)
    _, n = O.residual_norm(np.zeros((2, 8)), None, None, 1e-6, True)
    assert (n == 0).all()


@pytest.mark.parametrize("scoring", ["softmax", "sigmoid"])
@pytest.mark.parametrize("groups,top_groups", [(1, 1), (2, 1), (3, 2)])
def test_route_against_brute_force(scoring, groups, top_groups):
    """Every set of top_k experts of the kept groups: the chosen one has the largest sum of
    choices; the kept groups have the largest sum of ranks."""
    rng = np.random.default_rng(3)
    n, k = 6, 2
    logits, bias = rng.normal(size=(20, n)), 0.1 * rng.normal(size=n)
    ids, w, invalid, gap = O.route(logits, k, scoring, bias, groups, top_groups, scale=2.0)
    assert not invalid.any() and gap > 0
    for i in range(20):
        s = np.exp(logits[i]) / np.exp(logits[i]).sum() if scoring == "softmax" else \
            1 / (1 + np.exp(-logits[i]))
        c = s + bias
        size = n // groups
        rank = [sum(sorted(c[g * size:(g + 1) * size])[-2:]) for g in range(groups)]
        kept = max(itertools.combinations(range(groups), top_groups),
                   key=lambda gs: sum(rank[g] for g in gs))
        allowed = [e for e in range(n) if e // size in kept]
        best = max(itertools.combinations(allowed, k), key=lambda es: sum(c[e] for e in es))
        assert set(ids[i]) == set(best) and c[ids[i][0]] >= c[ids[i][1]]
        assert math.isclose(w[i].sum(), 2.0) and math.isclose(w[i][0] / w[i][1],
                                                             s[ids[i][0]] / s[ids[i][1]])


def test_route_ties_masks_and_bad_rows():
    inf = np.inf
    logits = np.array([[0.0, 0.0, 0.0, 0.0], [-inf, 1.0, -inf, 1.0], [-inf] * 4,
                       [0.0, np.nan, 0.0, 0.0], [inf, 0.0, 0.0, 0.0]])
    ids, w, invalid, _ = O.route(logits, 3, "softmax")
    assert ids[0].tolist() == [0, 1, 2] and np.allclose(w[0], 1 / 3)
    assert ids[1].tolist() == [1, 3, -1] and w[1].tolist() == [0.5, 0.5, 0.0]
    assert ids[2].tolist() == [-1, -1, -1] and (w[2] == 0).all()
    assert invalid.tolist() == [False, False, False, True, True] and (ids[3:] == -1).all()
    offsets, rows = O.plan(ids, 4)
    assert offsets.tolist() == [0, 1, 3, 4, 5]
    assert rows.tolist() == [0, 1, 3, 2, 4] + [-1] * 10


@pytest.mark.parametrize("mx", [True, False])
def test_experts_closed_form(mx):
    """One expert whose gate saturates: h = 64 u for g = 64, so y = w2 (64 w3 x) exactly."""
    d = f = 32
    x = np.zeros((2, d))
    x[0, 3], x[1, 7] = 1.0, -2.0
    w1 = np.zeros((1, f, d))
    w1[0, :, 3], w1[0, :, 7] = 64.0, -32.0
    w3 = np.zeros((1, f, d))
    w3[0, np.arange(f), 3] = 1.0
    w3[0, np.arange(f), 7] = 0.25
    w2 = np.eye(d)[None]
    y, tol = O.experts(x, w1, w3, w2, np.array([[0], [0]]), np.array([[0.5], [2.0]]), mx)
    assert np.allclose(y[0], 32.0, rtol=1e-12) and np.allclose(y[1], -64.0, rtol=1e-12)
    assert (tol < 1e-2).all()
    y, _ = O.experts(x, w1, w3, w2, np.array([[-1], [0]]), np.array([[0.5], [2.0]]), mx)
    assert (y[0] == 0).all()
