"""What the example stack refuses before it makes a call."""
import pytest
import torch

from paper_2603_09555_amd.hybrid import HybridConfig, HybridStack


def test_sequences_do_not_outgrow_their_pages():
    stack = HybridStack(HybridConfig(width=32, nheads=2, attn_heads=2, attn_kv_heads=1), torch.float32, device="cpu")
    cache = stack.new_cache(2, 20)     # two pages of 16 each
    with pytest.raises(ValueError, match="outgrown"):
        stack.prefill(torch.zeros(40, 32), [7, 33], cache)
    assert cache.held == [0, 0] and cache.lens.tolist() == [0, 0]
    cache.held, cache.lens = [32, 5], torch.tensor([32, 5], dtype=torch.int32)
    with pytest.raises(ValueError, match="outgrown"):
        stack.step(torch.zeros(2, 32), cache)
    assert cache.held == [32, 5] and cache.lens.tolist() == [32, 5]
    with pytest.raises(ValueError):
        stack.prefill(torch.zeros(3, 32), [3], cache)      # a length for every sequence
    cache.held = None                                      # (read from lens)
    with pytest.raises(ValueError, match="outgrown"):
        stack.step(torch.zeros(2, 32), cache)
    assert cache.held == [32, 5]
