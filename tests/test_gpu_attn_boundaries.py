"""Boundaries that decrease.  ssd.h promises nothing of the results then, but that nothing outside the tensors is touched; with
few sequences, those tokens that exactly one sequence counts are right all the same.  Limits as in test_gpu_attn.py."""
import pytest
import torch

from oracle import block_oracle
from parity import TOL, assert_close
from test_gpu_attn import TYPES, dev, make, ssd  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("io", ["f32", "bf16"])
@pytest.mark.parametrize("cu,alone", [([0, 10, 5, 70], [(0, 0, 5), (2, 10, 70)]), ([50, 0, 30, 60], [(1, 0, 30), (2, 30, 60)])])
def test_tokens_of_one_sequence(ssd, cu, alone, io):  # noqa: F811
    lengths = [90, 70, 80]
    s = make(lengths, 4, 2, 64, 16, io, new=[10, 40, 20], seed=37)
    s["cu"] = torch.tensor(cu, dtype=torch.int32)
    g = torch.Generator().manual_seed(38)
    k, v = (torch.randn((70, 2, 64), generator=g).to(TYPES[io]) for _ in range(2))
    d = dev(s)
    room = torch.full((72, 4, 64), 7.0, dtype=TYPES[io], device="cuda")
    ssd.ssd_attn_prefill(d["q"], d["k"], d["v"], d["table"], d["lens"], d["cu"], y=room[1:71])
    ssd.ssd_attn_append(None, k.cuda(), v.cuda(), d["k"], d["v"], d["table"], d["lens"], d["cu"])
    torch.cuda.synchronize()
    assert bool((room[0] == 7).all()) and bool((room[71] == 7).all())
    kept = torch.zeros_like(s["v"], dtype=torch.bool)
    for b in range(3):      # slots that some sequence may write
        for t in range(cu[b], max(cu[b], cu[b + 1])):
            pos = lengths[b] - (cu[b + 1] - t)
            if pos >= 0:
                kept[int(s["table"][b, pos // 16]), :, pos % 16] = True
    assert bool(((d["v"].cpu() == s["v"]) | (s["v"].isnan() & d["v"].cpu().isnan()) | kept).all())
    for b, lo, hi in alone:
        n = hi - lo
        ref = block_oracle.attention(s["q"][lo:hi], s["k"], s["v"], s["table"][b:b + 1], s["lens"][b:b + 1] - (cu[b + 1] - hi), torch.tensor([0, n]))
        assert_close(room[1 + lo:1 + hi], ref, TOL[io], "prefill")
        for t in range(lo, hi):
            pos = lengths[b] - (cu[b + 1] - t)
            assert torch.equal(d["v"][int(s["table"][b, pos // 16]), :, pos % 16].cpu(), v[t]), (b, t)
