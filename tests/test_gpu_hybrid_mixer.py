"""The packed convolution, the selective scan and the normed heads together, as the hybrid stack runs them: prompts in pieces and
then token by token against whole prompts, and a block's two calls against their fp64 oracle.

The same numbers are summed in other orders and by other kernels.  fp32: 1e-4 as for every kernel of the library.  bf16: a Mamba-1
block rounds its input, projection, convolution, step sizes (twice), B and C, output and projection, some eight roundings of
2^-8, as the other blocks do; four blocks and a final norm, with random signs: sqrt(36) x 2^-9 = 1.2e-2 on average, 5e-2 for the
largest of many."""
import numpy as np
import pytest
import torch

from oracle import mixer_oracle, ssd_oracle
from parity import assert_close

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("blocks", ["SSAS", "SMAM"])
@pytest.mark.parametrize("dtype,limit", [(torch.float32, 1e-4), (torch.bfloat16, 5e-2)], ids=["f32", "bf16"])
def test_tokens_continue_prompts(dtype, limit, blocks):
    from paper_2603_09555_amd import hybrid
    config = hybrid.HybridConfig(blocks=blocks, head_norm=True, residual_scale=0.5)
    print("hybrid", dtype, blocks, flush=True)
    assert hybrid.check(dtype, config=config) <= limit
    assert hybrid.check(dtype, lengths=(2, 2), steps=3, config=config, seed=3) <= limit
    # (three heads, states and channels of no round numbers)
    config = hybrid.HybridConfig(width=72, blocks=blocks, nheads=3, selective_states=10, head_norm=True, attn_heads=3, attn_kv_heads=1, attn_headdim=40,
                                 rotary=24)
    assert hybrid.check(dtype, lengths=(150, 1, 9), steps=2, config=config, seed=5) <= limit


def test_a_prompt_with_no_new_token_for_some():
    """Sequences without a token keep their states."""
    from paper_2603_09555_amd import hybrid
    stack = hybrid.HybridStack(hybrid.HybridConfig(blocks="SA", head_norm=True), torch.float32)
    cache = stack.new_cache(3, 64)
    g = torch.Generator().manual_seed(1)
    stack.prefill(torch.randn((30, 256), generator=g).cuda(), [10, 20, 0], cache)
    conv, state = cache.conv[0].clone(), cache.state[0].clone()
    stack.prefill(torch.randn((5, 256), generator=g).cuda(), [0, 4, 1], cache)
    assert torch.equal(cache.conv[0][0], conv[0]) and torch.equal(cache.state[0][0], state[0])
    assert not torch.equal(cache.conv[0][1], conv[1]) and not torch.equal(cache.state[0][2], state[2])


def test_convolution_and_scan_against_the_oracle():
    """Prompts through both calls, then tokens through both steps, states in place."""
    from paper_2603_09555_amd import ssd
    g = torch.Generator().manual_seed(2)
    C, N, lengths = 96, 16, [40, 0, 173]
    n = lambda *s: torch.randn(s, generator=g)   # noqa: E731
    T = sum(lengths)
    u, z, dt, bc = n(T, C), n(T, C), 0.5 * n(T, C), 0.5 * n(T, 2 * N + 3)
    w, b, A, D, bias = n(C, 4) / 4, 0.1 * n(C), -torch.rand((C, N), generator=g) * 8 - 0.5, n(C), 0.5 * n(C) - 3.0
    cu = torch.tensor([0] + lengths).cumsum(0).to(torch.int32)
    conv, state = n(3, C, 3), n(3, C, N)
    dc, ds = conv.cuda(), state.cuda()
    (x,), _ = ssd.ssd_conv1d_varlen(u.cuda(), w.cuda(), b.cuda(), cu.cuda(), dc, conv_state_out=dc)
    dbc = bc.cuda()
    rest = dict(dt_bias=bias.cuda(), dt_softplus=True)
    y, _ = ssd.ssd_selective_prefill(x, dt.cuda(), A.cuda(), dbc[:, 3:3 + N], dbc[:, 3 + N:], D.cuda(), cu.cuda(), z=z.cuda(), h0=ds, final_state=ds, **rest)
    xr, cr = mixer_oracle.conv1d_varlen(u, w, b, cu, conv)
    yr, sr = mixer_oracle.selective_scan(xr, ssd_oracle.dt_transform(dt, bias, True), A, bc[:, 3:3 + N], bc[:, 3 + N:], D, cu, z, state)
    assert_close(y, yr, 1e-4, "y")
    one = torch.arange(4, dtype=torch.int32)
    for _ in range(3):
        u, z, dt, bc = n(3, C), n(3, C), 0.5 * n(3, C), 0.5 * n(3, 2 * N)
        x, = ssd.ssd_conv1d_step(dc, u.cuda(), w.cuda(), b.cuda())
        y = ssd.ssd_selective_step(ds, x, dt.cuda(), A.cuda(), bc[:, :N].cuda(), bc[:, N:].cuda(), D.cuda(), z=z.cuda(), **rest)
        xr, cr = mixer_oracle.conv1d_varlen(u, w, b, one, cr)
        yr, sr = mixer_oracle.selective_scan(xr, ssd_oracle.dt_transform(dt, bias, True), A, bc[:, :N], bc[:, N:], D, one, z, sr)
        assert_close(y, yr, 1e-4, "y of a step")
    assert_close(ds, sr, 1e-4, "states")
    assert np.array_equal(dc.double().cpu().numpy(), cr)
