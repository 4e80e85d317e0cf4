"""Status words of the experts' MLP: a layer has one, and the decoding driver raises when a kernel
reports a failure in it: outputs that a wait which ran out left unwritten, and rows that the router
could not place, become no tokens."""
import numpy as np
import pytest
import torch

from paper_2608_26574_gb300 import binding as B
from paper_2608_26574_gb300 import decode as D
from paper_2608_26574_gb300.experts import ExpertMLP

pytestmark = pytest.mark.gpu


def _model(**kw):
    cfg = D.ModelConfig(vocab=256, d_model=256, n_layers=2, hq=2, hkv=2, head_dim=128, mlp=512,
                        logit_scale=8.0, **kw)
    return D.DLLM(cfg, seed=9)


def _decode(model, prompt=24):
    rng = np.random.default_rng(9)
    prompts = [rng.integers(0, 255, size=prompt).astype(np.int32) for _ in range(2)]
    return D.decode(model, prompts, 32, 16, thr=(0.01, 0.05), max_steps=40, min_progress=True)


def _short_waits(monkeypatch):
    """A short wait bound and a copy that is never issued (as the kernels' own failure tests)."""
    monkeypatch.setenv("DARD_TEST_WAIT_CYCLES", str(1 << 20))
    monkeypatch.setenv("DARD_TEST_DROP_KV", "1")


def test_a_wait_that_runs_out_in_the_experts_raises(monkeypatch):
    model = _model(experts=4, top_k=2)
    mlp = model.layers[1]["mlp"]

    def failing(h, delta=None):
        with monkeypatch.context() as m:
            _short_waits(m)
            return mlp(h, delta)

    model.layers[1]["mlp"] = failing
    with pytest.raises(RuntimeError, match="TIMEOUT"):
        _decode(model)
    model.layers[1]["mlp"] = mlp  # the next run starts with a clean word
    assert len(_decode(model)[1]) == 2


def test_a_wait_that_runs_out_in_the_attention_raises(monkeypatch):
    with monkeypatch.context() as m:
        _short_waits(m)
        with pytest.raises(RuntimeError, match="TIMEOUT"):
            _decode(_model(), prompt=300)  # several tiles of keys, the second of which is dropped


def test_a_row_that_the_router_cannot_place_raises():
    model = _model(experts=4, top_k=2)
    model.layers[0]["mlp"].router.fill_(float("nan"))
    with pytest.raises(RuntimeError, match="INVALID_ROW"):
        _decode(model)
    assert int(model.status.item()) != 0


def test_a_layer_without_a_status_word_has_its_own(monkeypatch):
    n, d, f = 4, 256, 512
    g = torch.Generator(device="cuda").manual_seed(1)
    w = [torch.randn(*s, generator=g, device="cuda") / 16 for s in ((n, f, d), (n, f, d), (n, d, f))]
    layer = ExpertMLP(*w, torch.randn(d, n, generator=g, device="cuda"), 2)
    h = torch.randn(20, d, generator=g, device="cuda")
    layer(h)
    assert int(layer.status.item()) == 0
    with monkeypatch.context() as m:
        _short_waits(m)
        layer(h)
    assert int(layer.status.item()) == B.STATUS_TIMEOUT
    layer.status.zero_()
    h[3, 5] = float("nan")
    layer(h)
    assert int(layer.status.item()) == B.STATUS_INVALID_ROW
