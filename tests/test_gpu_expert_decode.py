"""The experts' MLP as a layer (``experts.ExpertMLP``) and inside the decoding driver, on the GPU:
each operator's outputs against the float64 oracle on the inputs that it really had, and whole
blocks decoded by a model with experts."""
import numpy as np
import pytest
import torch

from oracle import mlp_oracle as O
from paper_2608_26574_gb300 import binding as B
from paper_2608_26574_gb300 import decode as D
from paper_2608_26574_gb300.experts import ExpertMLP

from .test_gpu_mlp import half_bf16

pytestmark = pytest.mark.gpu


def _np(t):
    return t.detach().double().cpu().numpy()


def _layer(dtype, mx, n, k, d, f, seed, **route):
    g = torch.Generator().manual_seed(seed)
    w = [torch.randn(*s, generator=g) / s[-1] ** 0.5 for s in ((n, f, d), (n, f, d), (n, d, f))]
    w = [t.cuda().to(dtype) for t in w]
    router = (torch.randn(d, n, generator=g) / d ** 0.5).cuda().to(dtype)
    return w, ExpertMLP(*w, router, k, mx=mx, route=route, status=torch.zeros(
        1, dtype=torch.int32, device="cuda"))


@pytest.mark.parametrize("dtype,mx", [(torch.bfloat16, True), (torch.bfloat16, False),
                                      (torch.float32, True)])
@pytest.mark.parametrize("tokens", [1, 75])
def test_layer_matches_the_oracle(dtype, mx, tokens):
    n, k, d, f = 12, 3, 128, 160
    bf16 = dtype == torch.bfloat16
    w, mlp = _layer(dtype, mx, n, k, d, f, tokens, scoring=B.ROUTE_SIGMOID, groups=3, top_groups=2)
    g = torch.Generator(device="cuda").manual_seed(2)
    h = torch.randn(tokens, d, generator=g, device="cuda").to(dtype)
    delta = torch.randn(tokens, d, generator=g, device="cuda").to(dtype)
    r, y = O.residual_norm(_np(h), _np(delta), None, 1e-6, bf16)
    out = mlp(h, delta)
    torch.cuda.synchronize()
    assert np.array_equal(_np(h), r)  # the residual, in place
    b = mlp._prepared(tokens)[0]
    half = half_bf16 if bf16 else np.zeros_like
    assert (np.abs(_np(b["y"]) - y) <= 4e-6 * np.abs(y) + half(y)).all()
    ids, wt, invalid, gap = O.route(_np(b["logits"]), k, "sigmoid", None, 3, 2)
    assert gap > 1e-6 and not invalid.any()
    assert np.array_equal(b["ids"].cpu().numpy(), ids)
    assert (np.abs(_np(b["weights"]) - wt) <= 4e-6 * wt).all()
    if mx:
        x = O.mx_value(_np(b["y8"]), b["y8_scale"].cpu().numpy()[:, :d // 32])
        wv = [O.mx_value(*O.mx_round(_np(t))) for t in w]
    else:
        x, wv = _np(b["y"]), [_np(t) for t in w]
    want, tol = O.experts(x, *wv, ids, _np(b["weights"]), mx)
    tol = tol + half(np.abs(want) + tol)
    assert (np.abs(_np(out) - want) <= tol).all()
    assert int(mlp.status.item()) == 0


def test_layers_share_workspaces_and_token_counts_come_and_go():
    shared: dict = {}
    g = torch.Generator(device="cuda").manual_seed(4)
    layers = []
    for seed in (1, 2):
        w, m = _layer(torch.bfloat16, True, 6, 2, 64, 96, seed)
        layers.append(ExpertMLP(*w, m.router, 2, workspaces=shared))
    hs = {t: torch.randn(t, 64, generator=g, device="cuda").to(torch.bfloat16) for t in (3, 40)}
    first = {(i, t): m(hs[t]).clone() for t in hs for i, m in enumerate(layers)}
    assert len(shared) == 2
    for (i, t), want in first.items():
        assert torch.equal(layers[i](hs[t]), want)


@pytest.mark.parametrize("mx", [True, False])
def test_decode_with_experts(mx):
    """Blocks reach all-U under low thresholds (as the dense model's test), the generated tokens
    hold no mask token, and no status bit is set."""
    cfg = D.ModelConfig(vocab=512, d_model=256, n_layers=2, hq=2, hkv=2, head_dim=128, mlp=192,
                        logit_scale=8.0, experts=8, top_k=2, expert_mx=mx)
    model = D.DLLM(cfg, seed=5)
    rng = np.random.default_rng(5)
    prompts = [rng.integers(0, cfg.vocab - 1, size=40).astype(np.int32) for _ in range(3)]
    gen, steps, us, _ = D.decode(model, prompts, 64, 32, thr=(0.01, 0.05), max_steps=96,
                                 min_progress=True)
    assert len(steps) == 2 and all(1 <= s < 96 for s in steps)
    assert not (gen == cfg.mask_token).any()
    assert int(model.status.item()) == 0


def test_one_expert_is_the_dense_mlp():
    """A dense fp32 model and one with a single expert of the same weights: the logits differ by
    the MXFP8 rounding of the MLP's products alone. Two roundings of 2^-4 at most per product
    move the MLP's output by a few percent of itself, far below its size."""
    kw = dict(vocab=256, d_model=256, n_layers=2, hq=2, hkv=2, head_dim=64, mlp=256, dtype="f32")
    dense = D.DLLM(D.ModelConfig(**kw), seed=3)
    one = D.DLLM(D.ModelConfig(**kw, experts=1, top_k=1), seed=3)
    for a, b in zip(dense.layers, one.layers):
        for n in ("wq", "wk", "wv", "wo"):
            b[n] = a[n]
        b["mlp"] = ExpertMLP(a["w1"].T[None].contiguous(), a["w3"].T[None].contiguous(),
                             a["w2"].T[None].contiguous(), b["mlp"].router, 1, status=one.status)
    one.emb, one.head = dense.emb, dense.head
    rng = np.random.default_rng(3)
    prompts = [rng.integers(0, 255, size=n).astype(np.int32) for n in (24, 17)]
    lx, ls = (_np(t) for t in dense.forward(D.make_batch(prompts, 32, 16, 0, None, dense.cfg, "cuda")))
    mx, ms = (_np(t) for t in one.forward(D.make_batch(prompts, 32, 16, 0, None, one.cfg, "cuda")))
    for a, b in ((lx, mx), (ls, ms)):
        assert np.linalg.norm(a - b) < 0.1 * np.linalg.norm(a)
        assert np.linalg.norm(a - b) > 0
