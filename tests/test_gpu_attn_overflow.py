"""Logits that fp32 does not hold give y that is not a number, as the formula in fp32 does, and no zeros as if nothing were seen."""
import pytest
import torch

from test_gpu_attn import make, run_prefill, run_step, ssd  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("io", ["f32", "bf16"])
@pytest.mark.parametrize("heads", [(4, 2, 64, 16), (2, 1, 128, 16), (1, 1, 256, 16)], ids=lambda h: "x".join(map(str, h)))
def test_logits_beyond_fp32(ssd, heads, io):  # noqa: F811
    for more in (0, -(-600000 // heads[2] // 16)):
        s = make([70, 300], *heads, io, new=[30, 40], seed=90, more_pages=more)
        s["q"] *= 1e18
        s["k"] *= 1e10
        # the scores, 1e28 and more, are numbers: their products with the scale, 1e40 where they are positive, are not
        y = run_prefill(ssd, s, scale=1e12)
        rows = s["q"].float().abs().amax(dim=2) > 0
        assert not torch.isfinite(y).any(dim=2).cpu()[rows].any()
        one = dict(s, q=s["q"][:2].contiguous())
        assert not torch.isfinite(run_step(ssd, one, scale=1e12)).any()
        # (the same scores, and a scale that they can have)
        assert torch.isfinite(run_prefill(ssd, s, scale=1e-28)).all() and torch.isfinite(run_step(ssd, one, scale=1e-28)).all()
