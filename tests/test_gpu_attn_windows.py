"""Windows as wide as a sequence's row of the page table and wider are no limit, to the last one that an int32 holds and beyond."""
import pytest
import torch

from test_gpu_attn import make, run_prefill, run_step, ssd  # noqa: F401

WIDE = [2 ** 31 - 1, 2 ** 31 - 2, 2 ** 30, 2 ** 32 + 5, 2 ** 63]


@pytest.mark.gpu
@pytest.mark.parametrize("io", ["f32", "bf16"])
def test_wide_windows(ssd, io):  # noqa: F811
    """Also where a unit begins with tokens in front of its sequence's beginning."""
    s = make([70, 200], 4, 2, 64, 16, io, new=[100, 60], seed=5)
    capacity = s["table"].shape[1] * 16
    y = run_prefill(ssd, s)
    assert bool((y[:30] == 0).all()) and bool((y[30:100].abs().amax(dim=(1, 2)) > 0).all())
    for window in [capacity, capacity + 1] + WIDE:
        assert torch.equal(run_prefill(ssd, s, window=window), y), window
    assert not torch.equal(run_prefill(ssd, s, window=capacity - 50), y)
    s["q"] = s["q"][:2].contiguous()
    ys = run_step(ssd, s)
    for window in [capacity, capacity + 1] + WIDE:
        assert torch.equal(run_step(ssd, s, window=window), ys), window


def test_shapes_hold_windows_that_an_int32_does_not():
    from paper_2603_09555_amd import ssd as binding
    cache, table = torch.zeros(5, 2, 16, 64), torch.zeros(3, 4, dtype=torch.int32)
    for window in WIDE:
        assert binding.make_attn_shape(3, 3, 4, cache, table, window).window == min(window, 2 ** 31 - 1)
    for window in (-1, -2 ** 31, -2 ** 32 + 5):
        assert binding.make_attn_shape(3, 3, 4, cache, table, window).window < 0
    assert binding.make_attn_shape(3, 3, 4, cache, table, 7).window == 7
