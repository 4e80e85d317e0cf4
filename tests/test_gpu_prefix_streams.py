"""``prefix.PrefixCache`` on streams and devices other than those of its making."""
import pytest
import torch

from paper_2608_26574_gb300 import binding as B
from paper_2608_26574_gb300.prefix import PrefixCache

from . import test_gpu_prefix_cache as C

pytestmark = pytest.mark.gpu
DEV = "cuda"


def test_cache_is_on_one_device():
    """"cuda" is the device that is current when the cache is made, not at each later call."""
    c = PrefixCache(1, 4, 2, 64, 10)
    assert c.device == torch.device("cuda", torch.cuda.current_device())
    assert c._scratch(16).device == c.keys(0).device == c.device


def test_workspace_of_a_call_on_another_stream():
    """A prepared attention runs on another stream and is dropped while it is still in flight there: its
    workspace is not handed out again meanwhile."""
    c, g = C._filled(layers=1, n=3000, capacity=3000)
    q = torch.randn(3, 8, 64, generator=g, device=DEV).to(torch.bfloat16)
    k, v = (torch.randn(3, 2, 64, generator=g, device=DEV).to(torch.bfloat16) for _ in range(2))
    want, o = torch.empty_like(q), torch.empty_like(q)
    call = c.attention([3], [0], [0], [0], None, None, None)
    c.attend(call, 0, q, k, v, want)
    torch.cuda.synchronize()
    size, at = call._scratch[1], call._scratch[0]
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        torch.cuda._sleep(100_000_000)  # some 50 ms
        c.attend(call, 0, q, k, v, o)
    del call
    others = [torch.empty(size, dtype=torch.uint8, device=DEV) for _ in range(3)]  # (left unwritten)
    busy = not side.query()
    assert busy and all(x.data_ptr() != at for x in others)
    side.synchronize()
    assert torch.equal(o, want)


def test_calls_that_the_cache_did_not_prepare():
    """``attend`` takes any ``PrefixAttentionCall``, with its own workspace or none, and a graph may capture one
    that was prepared on another stream."""
    c, g = C._filled(layers=1, n=3000, capacity=3000)
    q = torch.randn(3, 8, 64, generator=g, device=DEV).to(torch.bfloat16)
    k, v = (torch.randn(3, 2, 64, generator=g, device=DEV).to(torch.bfloat16) for _ in range(2))
    want, o, plain = (torch.empty_like(q) for _ in range(3))
    call = c.attention([3], [0], [0], [0], None, None, None)
    c.attend(call, 0, q, k, v, want)
    ws = torch.empty(call._scratch[1], dtype=torch.uint8, device=DEV)
    c.attend(B.PrefixAttentionCall([3], [0], [0], [0], None, None, None, workspace=ws), 0, q, k, v, o)
    assert torch.equal(o, want)
    c.attend(B.PrefixAttentionCall([3], [0], [0], [0], None, None, None), 0, q, k, v, plain)
    assert (plain.float() - want.float()).abs().max() <= 2 ** -6 * want.float().abs().max()
    o.zero_()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        c.attend(call, 0, q, k, v, o)
    for _ in range(3):
        graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(o, want)
