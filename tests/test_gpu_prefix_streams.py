"""``prefix.PrefixCache`` on streams and devices other than those of its making."""
import pytest
import torch

from paper_2608_26574_gb300.prefix import PrefixCache

pytestmark = pytest.mark.gpu

def test_cache_is_on_one_device():
    """"cuda" is the device that is current when the cache is made, not at each later call."""
    c = PrefixCache(1, 4, 2, 64, 10)
    assert c.device == torch.device("cuda", torch.cuda.current_device())
    assert c._scratch(16).device == c.keys(0).device == c.device
