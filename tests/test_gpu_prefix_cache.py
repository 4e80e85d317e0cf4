"""The prefix cache of a model (``prefix.PrefixCache``) and decoding behind a shared prefix."""
import numpy as np
import pytest
import torch

from oracle import prefix_oracle as O
from paper_2608_26574_gb300 import binding as B
from paper_2608_26574_gb300 import decode as D
from paper_2608_26574_gb300.prefix import PrefixCache

pytestmark = pytest.mark.gpu
DEV = "cuda"


def _np(t):
    return t.double().cpu().numpy()


def _filled(layers=3, hq=8, hkv=2, d=64, n=300, capacity=330, dtype=torch.bfloat16):
    c = PrefixCache(layers, hq, hkv, d, capacity, dtype)
    g = torch.Generator(DEV).manual_seed(3)
    for i in range(layers):
        c.store(i, *(torch.randn(n, hkv, d, generator=g, device=DEV).to(dtype) for _ in range(2)))
    return c, g


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_cache_accumulates_and_evicts_by_layer(dtype):
    c, g = _filled(dtype=dtype)
    want_w = []
    for i in range(3):
        total = None
        for step in range(2):
            q = torch.randn(11, 8, 64, generator=g, device=DEV).to(dtype)
            lse = torch.full((11, 8), 6.0 + step, device=DEV)
            c.accumulate(i, q, lse)
            total = O.prefix_weights(_np(q), _np(lse), _np(c.keys(i)), total, 1.0)[0]
        assert np.allclose(_np(c.weights(i)), total, rtol=1e-4)
        want_w.append(_np(c.weights(i)))
    old = [(c.keys(i).clone(), c.values(i).clone()) for i in range(3)]
    c.evict(100, 4, 10)
    heads = torch.arange(2, device=DEV)[:, None]
    for i in range(3):
        kept = torch.from_numpy(O.prefix_evict(want_w[i], 100, 4, 10)).long().to(DEV)
        assert c.length(i) == 100 and c.start == 300
        assert torch.equal(c.keys(i), old[i][0][kept, heads].transpose(0, 1))
        assert torch.equal(c.values(i), old[i][1][kept, heads].transpose(0, 1))
        assert np.array_equal(_np(c.weights(i)), np.take_along_axis(want_w[i], kept.cpu().numpy(), 1))
    c.evict(100)  # nothing to do
    assert c.length() == 100
    c.evict(0)
    assert c.length(2) == 0 and c.weights(2).shape == (2, 0)
    c.accumulate(0, torch.zeros(1, 8, 64, device=DEV, dtype=dtype), torch.zeros(1, 8, device=DEV))


def test_cache_attention_after_eviction():
    """A call prepared once serves every layer, before and after an eviction."""
    c, g = _filled()
    q = torch.randn(5, 8, 64, generator=g, device=DEV).to(torch.bfloat16)
    k, v = (torch.randn(5, 2, 64, generator=g, device=DEV).to(torch.bfloat16) for _ in range(2))
    call = c.attention([2, 3], [0, 0], [0, 0], [0, 0], None, None, None)
    from oracle import dard_oracle as DO
    none = lambda n: DO.SeqLayout(n, 0, np.zeros(0, np.uint8), np.zeros(0, np.float32),  # noqa: E731
                                  np.zeros(0, np.int32))
    for keep in (300, 77, 0):
        c.evict(keep)
        for i in range(3):
            o, lse = torch.empty_like(q), torch.empty(5, 8, device=DEV)
            c.attend(call, i, q, k, v, o, lse)
            want, wl, mass, _ = O.prefix_attention(*(_np(x) for x in (q, k, v, c.keys(i), c.values(i))),
                                                   [none(2), none(3)])
            assert (np.abs(_np(o) - want) <= mass * 2.0 ** -7 * 1.02 + np.abs(want) * 2.0 ** -8 + 1e-6).all()
            assert np.abs(_np(lse) - wl).max() < 1e-4


def test_cache_graphs_side_by_side():
    """Two captured steps, in parts, replayed on two streams at once: each has its own workspaces."""
    c, g = _filled(layers=2, hq=8, hkv=2, n=3000, capacity=3000)
    steps = []
    for i in range(2):
        q = torch.randn(3, 8, 64, generator=g, device=DEV).to(torch.bfloat16)
        k, v = (torch.randn(3, 2, 64, generator=g, device=DEV).to(torch.bfloat16) for _ in range(2))
        steps.append((q, k, v, torch.empty_like(q), torch.empty(3, 8, device=DEV)))

    def step(i):
        q, k, v, o, lse = steps[i]
        call = c.attention([3], [0], [0], [0], None, None, None)
        c.attend(call, i, q, k, v, o, lse)
        c.accumulate(i, q, lse, decay=0.0)
        return call

    want, graphs, calls = [], [], []
    for i in range(2):
        step(i)
        want.append([x.clone() for x in (*steps[i][3:], c.weights(i))])
    torch.cuda.synchronize()
    for i in range(2):
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            calls.append(step(i))
    assert calls[0]._scratch[0] != calls[1]._scratch[0]
    streams = [torch.cuda.Stream() for _ in range(2)]
    for _ in range(50):
        for graph, stream in zip(graphs, streams):
            with torch.cuda.stream(stream):
                graph.replay()
    torch.cuda.synchronize()
    for i in range(2):
        assert all(torch.equal(a, b) for a, b in zip(want[i], (*steps[i][3:], c.weights(i))))


def test_cache_refusals():
    c, _ = _filled()
    z = torch.zeros(5, 2, 64, device=DEV, dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="expected, got"):
        c.store(0, z[:, :1], z[:, :1])
    with pytest.raises(ValueError, match="expected, got"):
        c.store(0, z.new_zeros(331, 2, 64), z.new_zeros(331, 2, 64))
    with pytest.raises(ValueError, match="keep"):
        c.evict(5, 3, 3)
    with pytest.raises(ValueError, match="keep_first|keep -1|keep"):
        c.evict(-1)


@pytest.mark.parametrize("experts", [0, 4])
def test_forward_behind_a_prefix(experts):
    """With one layer the prefix's keys and values depend on its own tokens alone, so that the
    forward pass over the cache gives what the pass over whole sequences gives."""
    cfg = D.ModelConfig(vocab=128, d_model=128, n_layers=1, hq=4, hkv=2, head_dim=64, mlp=128, dtype="f32"
                        if not experts else "bf16", experts=experts, expert_mx=False)
    model = D.DLLM(cfg, seed=2)
    rng = np.random.default_rng(0)
    shared = rng.integers(0, 127, 150).astype(np.int32)
    own = [rng.integers(0, 127, n).astype(np.int32) for n in (3, 0, 40)]
    whole = D.make_batch([np.concatenate([shared, x]) for x in own], 16, 8, 1, None, cfg, DEV)
    part = D.make_batch(own, 16, 8, 1, None, cfg, DEV)
    for b in (whole, part):
        b.state.copy_(torch.arange(24, device=DEV) % 3)
        b.prev_conf.copy_(torch.linspace(0.1, 0.9, 24, device=DEV))
    lx, ls = model.forward(whole)
    cache = model.cache_prefix(shared)
    px, ps = model.forward(part, prefix=cache, weigh=True)
    scale = lx.abs().max().item()
    # fp32: sums of 128 and 150 terms in two orders; bf16: a handful of roundings of 2^-8 each
    lim = (2e-5 if not experts else 0.06) * scale
    assert (lx.float() - px.float()).abs().max().item() <= lim
    assert (ls.float() - ps.float()).abs().max().item() <= lim
    # the probabilities of every row of the batch: what they left for the prefix, at most 1 a row
    rows = part.tokens.numel()
    total = cache.weights(0).sum(1) / 2  # heads of the group
    assert ((total > 0) & (total < rows)).all()


def test_forward_rows_without_output_add_no_weight():
    """Shadow rows with a repeated source are not stored, and add nothing to the keys' weights."""
    cfg = D.ModelConfig(vocab=128, d_model=128, n_layers=1, hq=4, hkv=2, head_dim=64, mlp=128)
    model = D.DLLM(cfg, seed=2)
    rng = np.random.default_rng(0)
    prefix = model.cache_prefix(rng.integers(0, 127, 150).astype(np.int32))
    batch = D.make_batch([rng.integers(0, 127, 5).astype(np.int32)], 16, 8, 0, None, cfg, DEV)
    batch.shadow_src[2:] = batch.shadow_src[1]
    rows = batch.tokens.numel()
    for _ in range(8):  # what the allocator hands out next is no number
        torch.full((rows, cfg.hq), torch.nan, device=DEV)
    model.forward(batch, prefix=prefix, weigh=True)
    w = prefix.weights(0)
    assert torch.isfinite(w).all() and (w >= 0).all()
    # every stored row (all but six) spends at most a weight of 1 per head
    assert float(w.sum()) <= (rows - 6) * cfg.hq * (1 + 1e-3)


@pytest.mark.parametrize("keep", [0, 40])
def test_decode_behind_a_prefix(keep):
    cfg = D.ModelConfig(vocab=128, d_model=128, n_layers=2, hq=4, hkv=2, head_dim=64, mlp=128,
                        logit_scale=8.0)
    model = D.DLLM(cfg, seed=5)
    rng = np.random.default_rng(1)
    shared = rng.integers(0, 127, 100).astype(np.int32)
    prompts = [rng.integers(0, 127, n).astype(np.int32) for n in (4, 9)]
    caches = []
    make = model.cache_prefix
    model.cache_prefix = lambda t: caches.append(make(t)) or caches[-1]
    gen, steps, _, _ = D.decode(model, prompts, 24, 8, max_steps=12, min_progress=True, shared=shared,
                                keep=keep, keep_ends=(2, 8))
    assert gen.shape == (2, 24) and (gen != cfg.mask_token).all() and len(steps) == 3
    assert [caches[0].length(i) for i in range(2)] == [keep or 100] * 2
    again, _, _, _ = D.decode(model, prompts, 24, 8, max_steps=12, min_progress=True, shared=shared,
                              keep=keep, keep_ends=(2, 8))
    assert np.array_equal(gen, again)


def test_decode_refusals():
    model = D.DLLM(D.ModelConfig(vocab=64, d_model=128, n_layers=1, hq=2, hkv=2, head_dim=64, mlp=64))
    p = [np.arange(4, dtype=np.int32)]
    with pytest.raises(ValueError, match="shared"):
        D.decode(model, p, 8, 8, keep=5)
    with pytest.raises(ValueError, match="ends"):
        D.decode(model, p, 8, 8, shared=p[0], keep=5)
