"""The hybrid stack of paper_2603_09555_amd.hybrid: prompts in pieces and then token by token against whole prompts.

The same numbers are summed in other orders and by other kernels.  fp32: 1e-4 as for every kernel of the library.  bf16: a
block rounds its input, projections, core, norm and output, some eight roundings of 2^-8 that fall differently where fp32 sums
differ; four blocks and a final norm, with random signs: sqrt(36) x 2^-9 = 1.2e-2 on average, 5e-2 for the largest of many."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("window", [0, 48])
@pytest.mark.parametrize("dtype,limit", [(torch.float32, 1e-4), (torch.bfloat16, 5e-2)], ids=["f32", "bf16"])
def test_tokens_continue_prompts(dtype, limit, window):
    from paper_2603_09555_amd import hybrid
    config = hybrid.HybridConfig(window=window, residual_scale=0.5)
    print("hybrid", dtype, window, flush=True)
    assert hybrid.check(dtype, config=config) <= limit
    assert hybrid.check(dtype, lengths=(2, 2), steps=3, config=config, seed=3) <= limit
