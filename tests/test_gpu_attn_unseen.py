"""Values that are not finite, of a sequence's own tokens, out of a row's sight: from 96 tokens (fp32: 64) on from what the row
sees they don't matter to ssd_attn_prefill, nor any to a row that sees nothing, and to ssd_attn_step none that its row does not see.
Limits as in test_gpu_attn.py."""
import numpy as np
import pytest
import torch

from oracle import block_oracle
from parity import TOL, assert_close
from test_gpu_attn import make, run_prefill, run_step, ssd  # noqa: F401

pytestmark = pytest.mark.gpu
HEADS = [(2, 2, 64, 16), (4, 2, 128, 16), (4, 1, 128, 64), (1, 1, 256, 16), (3, 3, 80, 8), (2, 1, 200, 16)]
FAR = {"f32": 64, "bf16": 96}
PIECES = [([200], [33]), ([150, 90], [63, 0]), ([300, 40], [0, -20])]      # new tokens, cached tokens (negative: no place for all)


def spoil(s, b, token, page):
    """A token's values, of all key heads, become infinite and NaN."""
    where = int(s["table"][b, token // page])
    s["v"][where, :, token % page, ::2] = float("inf")
    s["v"][where, :, token % page, 1::2] = float("nan")


@pytest.mark.parametrize("io", ["f32", "bf16"])
@pytest.mark.parametrize("heads", HEADS, ids=lambda h: "x".join(map(str, h)))
def test_prefill(ssd, heads, io):  # noqa: F811
    for i, (new, prior) in enumerate(PIECES):
        lengths = [a + b for a, b in zip(new, prior)]
        clean = make(lengths, *heads, io, new=new, seed=20 + i)
        for window in (0, 1, 64, 100):
            ref = block_oracle.attention(clean["q"], clean["k"], clean["v"], clean["table"], clean["lens"], clean["cu"], window=window)
            for token in (0, 31, 32, 64, 127, 128, lengths[0] - 1):
                s = dict(clean, v=clean["v"].clone())
                spoil(s, 0, token, heads[3])
                print("prefill", heads, io, new, prior, window, token, flush=True)
                y = run_prefill(ssd, s, window=window).cpu()
                pos = prior[0] + np.arange(new[0])
                first = np.maximum(pos - window + 1, 0) if window else np.zeros_like(pos)
                far = (token - pos >= FAR[io]) | (first - token >= FAR[io]) | (pos < 0)
                rows = np.concatenate([np.nonzero(far)[0], np.arange(new[0], len(ref))])     # and the other sequence's
                if len(rows):
                    assert_close(y[rows], ref[rows], TOL[io], "prefill")
                seen = (first <= token) & (token <= pos)
                assert not torch.isfinite(y[:new[0]][torch.tensor(seen)]).any(), "what is seen shows"


@pytest.mark.parametrize("io", ["f32", "bf16"])
def test_prefill_without_a_place(ssd, io):  # noqa: F811
    """Rows in front of a sequence's beginning, and behind its row of the table, beside rows that see what is not finite."""
    s = make([40, 64], 1, 1, 64, 16, io, new=[100, 50], seed=30)
    s["lens"][1] += 30
    for b, token in ((0, 0), (0, 39), (1, 44), (1, 63)):
        spoil(s, b, token, 16)
    y = run_prefill(ssd, s).cpu()
    assert bool((y[:60] == 0).all()) and bool((y[120:] == 0).all())
    assert not torch.isfinite(y[60:100]).any()


@pytest.mark.parametrize("io", ["f32", "bf16"])
def test_prefill_shared_units(ssd, io):  # noqa: F811
    """Parts of units, in most of which a row of a window sees nothing."""
    clean = make([5000], 8, 1, 128, 16, io, new=[20], seed=31)
    for token, window in ((0, 3000), (1900, 3000), (3000, 1500), (4979, 0)):
        ref = block_oracle.attention(clean["q"], clean["k"], clean["v"], clean["table"], clean["lens"], clean["cu"], window=window)
        s = dict(clean, v=clean["v"].clone())
        spoil(s, 0, token, 16)
        y = run_prefill(ssd, s, window=window)
        if token == 4979:
            assert not torch.isfinite(y).any()
        else:
            assert_close(y, ref, TOL[io], "prefill")


@pytest.mark.parametrize("io", ["f32", "bf16"])
def test_step(ssd, io):  # noqa: F811
    for more in (0, 9000):
        clean = make([300, 77], 4, 2, 128, 16, io, seed=32, more_pages=more)
        for window in (1, 64, 65):
            ref = block_oracle.attention(clean["q"], clean["k"], clean["v"], clean["table"], clean["lens"], window=window)
            s = dict(clean, v=clean["v"].clone(), k=clean["k"].clone())
            spoil(s, 0, 300 - window - 1, 16)
            s["k"][int(s["table"][1, 0])] = float("nan")
            y = run_step(ssd, s, window=window)
            rows = [0, 1] if window < 62 else [0]      # (a wider window reaches the second sequence's first page)
            assert_close(y[rows], ref[rows], TOL[io], "step")
