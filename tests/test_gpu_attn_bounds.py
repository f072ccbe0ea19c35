"""Attention over a paged cache at the limits of its arithmetic, so that a lost part of it shows.

bf16.  A product of two bf16 values is exact in fp32.  A probability is rounded to bf16, and y is: relative errors of the same
distribution.  y = sum p v of values of no common sign has the size of sqrt(sum p^2 v^2), which is also what the probabilities'
errors add up by, so that they make an error like y's own rounding; together sqrt(2) of it, and a little more where the sum of the
probabilities has them too.  Limit: twice the root mean square of the exact result's rounding to bf16, over all of a call's y.

fp32.  An exponent is a sum of headdim products; each is off by 2^-24 at most, and so is each of the sum's partial results, of
size 12 at most here (logits of deviation 2): with random signs sqrt(2 x 256) x 2^-24 x 12 / 2 = 8e-6 at headdim 256 if all of
them were that large, half of it if they grow evenly; its scaling and the maximum's subtraction, one rounding of up to 32 each,
2e-6; the hardware's exponential and the products' sums 1e-6.  So a probability, and |error| / sum p |v|, is off by 1e-5 at most."""
import math

import numpy as np
import pytest
import torch

from oracle import block_oracle
from parity import to_np64
from test_gpu_attn import make, run_prefill, run_step, ssd  # noqa: F401

pytestmark = pytest.mark.gpu
HEADS = [(4, 2, 64, 16), (32, 8, 128, 16), (5, 1, 64, 64), (14, 2, 80, 32), (2, 2, 256, 16), (33, 1, 112, 16)]


def within(got, s, cu, io, what, **kw):
    ref = block_oracle.attention(s["q"], s["k"], s["v"], s["table"], s["lens"], cu, **kw)
    mag = block_oracle.attention(s["q"], s["k"], s["v"].abs(), s["table"], s["lens"], cu, **kw)
    limit = 1e-5 * mag + 2.0 ** -24 * np.abs(ref)
    g = to_np64(got)
    assert np.isfinite(g).all(), what
    if io == "bf16":
        rms = lambda e: float(np.sqrt(np.mean(e * e)))     # noqa: E731
        own = rms(to_np64(torch.tensor(ref).bfloat16()) - ref)
        print("%s %s: %.2f of the result's own rounding" % (what, io, rms(g - ref) / own), flush=True)
        assert rms(g - ref) <= 2 * own, (what, rms(g - ref) / own)
        return
    ratio = np.abs(g - ref) / np.where(limit > 0, limit, 1.0)
    print("%s %s: %.2f of the limit at most" % (what, io, ratio.max()), flush=True)
    assert (np.abs(g - ref) <= limit).all(), (what, ratio.max())


@pytest.mark.parametrize("io", ["f32", "bf16"])
@pytest.mark.parametrize("heads", HEADS, ids=lambda h: "x".join(map(str, h)))
def test_step(ssd, heads, io):  # noqa: F811
    for more in (0, -(-600000 // heads[2] // heads[3])):    # (a unit to a workgroup, and dealt)
        s = make([1, 33, 700, 2049], *heads, io, seed=80, more_pages=more)
        for window in (0, 40):
            within(run_step(ssd, s, window=window), s, None, io, "step", window=window)


@pytest.mark.parametrize("io", ["f32", "bf16"])
@pytest.mark.parametrize("heads", HEADS, ids=lambda h: "x".join(map(str, h)))
def test_prefill(ssd, heads, io):  # noqa: F811
    for new, prior in (([260], [0]), ([7, 70], [1000, 513]), ([3], [4000])):
        s = make([a + b for a, b in zip(new, prior)], *heads, io, new=new, seed=81)
        for window in (0, 50):
            within(run_prefill(ssd, s, window=window), s, s["cu"], io, "prefill", window=window)


def few(D, tokens, rows):
    """One sequence of ``tokens`` tokens behind which ``rows`` tokens are new and see all of these (their own keys weigh nothing)."""
    page = 16
    pages = -(-(tokens + rows) // page)
    k = torch.zeros(pages, 1, page, D)
    v = torch.zeros(pages, 1, page, D)
    return dict(q=torch.zeros(rows, 1, D), k=k, v=v, table=torch.arange(pages, dtype=torch.int32)[None],
                lens=torch.tensor([tokens + rows], dtype=torch.int32), cu=torch.tensor([0, rows], dtype=torch.int32))


@pytest.mark.parametrize("D", [64, 128, 256])
def test_one_token_is_its_value(ssd, D):  # noqa: F811
    """Softmax over one token: y is its value, to a few roundings -- each of its 24 bits is in the product."""
    g = torch.Generator().manual_seed(82)
    s = few(D, 0, 40)
    s["q"], s["k"] = torch.randn(40, 1, D, generator=g), torch.randn(s["k"].shape, generator=g)
    s["v"] = torch.randn(s["v"].shape, generator=g)
    own = s["v"].view(-1, D)[:40]
    for y in (run_prefill(ssd, s, window=1),
              run_step(ssd, dict(s, q=s["q"], table=s["table"].expand(40, -1).contiguous(), lens=torch.arange(1, 41, dtype=torch.int32)), window=1)):
        err = ((y.view(40, D).cpu().double() - own.double()).abs() / own.double().abs()).max().item()
        assert err <= 6 * 2.0 ** -24, err     # p, its part of the sum, the reciprocal, two products and their sum


@pytest.mark.parametrize("D", [64, 128, 256])
def test_equal_values_are_y(ssd, D):  # noqa: F811
    """All values equal: y is that value whatever the probabilities are, if these go whole into both sums."""
    g = torch.Generator().manual_seed(83)
    for tokens in (2, 3, 30):
        s = few(D, tokens, 64)
        s["q"] = 2 * torch.randn(64, 1, D, generator=g)
        s["k"] = torch.randn(s["k"].shape, generator=g)
        s["v"][:] = torch.randn(D, generator=g)
        want = s["v"][0, 0, 0].double()
        y = run_prefill(ssd, s).view(64, D).cpu().double()
        # (sums of up to 94 terms in another order each: 2^-24 x sqrt(94) x a few)
        assert ((y - want).abs() / want.abs()).max().item() <= 40 * 2.0 ** -24, tokens


LO = 2.0 ** -20      # of 1 + 2^-9 + 2^-20 the last of three bf16 parts


@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("what", ["key", "query", "middles"])
def test_small_parts_of_a_product_count(ssd, D, what):  # noqa: F811
    """Two tokens whose scores differ by what one product of small parts gives, enlarged to a logit of 1: the weights are
    e / (1 + e) and 1 / (1 + e).  The products are exact in fp32.  The new tokens' own keys are far below."""
    s = few(D, 2, 8)
    k, q, v = s["k"].view(-1, D), s["q"].view(-1, D), s["v"].view(-1, D)
    at = min(D - 1, 37)
    if what == "key":        # q = 1, k = 1 + 2^-9 + 2^-20 and 1 + 2^-9
        q[:, at] = 1.0
        k[0, at], k[1, at], scale = 1 + 2.0 ** -9 + LO, 1 + 2.0 ** -9, 1 / LO
    elif what == "query":    # the same of q, in two places, at each of which one key is 1
        q[:, at], q[:, 3] = 1 + 2.0 ** -9 + LO, 1 + 2.0 ** -9
        k[0, at], k[1, 3], scale = 1.0, 1.0, 1 / LO
    else:                    # (1 + 2^-9)^2 = 1 + 2^-8 + 2^-18, and 1 + 2^-8
        q[:, at], q[:, 3] = 1 + 2.0 ** -9, 1.0
        k[0, at], k[1, 3], scale = 1 + 2.0 ** -9, 1 + 2.0 ** -8, 2.0 ** 18
    k[2:, 5], q[:, 5] = -1.0, 1.0
    v[0], v[1], v[2:] = 1.0, -1.0, 100.0
    want = (math.e - 1) / (math.e + 1)
    one = dict(s, q=s["q"][:1].contiguous(), lens=torch.tensor([3], dtype=torch.int32))
    for name, y in (("prefill", run_prefill(ssd, s, scale=scale)), ("step", run_step(ssd, one, scale=scale))):
        # an exponent is one rounding of a difference of size 1.4
        assert (y.double().cpu() - want).abs().max().item() <= 1e-6, name
