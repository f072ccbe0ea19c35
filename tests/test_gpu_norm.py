"""GPU parity of the norms on either side of a block against the fp64 oracle, element by element.

Limits: an output in bf16 is rounded once, at most 2^-8 of its value (8 significant bits).  In front of that, fp32: a sum of
squares of positive terms over chains of at most 32 and a tree (32 + 10 roundings of 2^-24, halved by the root), silu with
an exponent rounded at |z| up to about 8 (8 x 2^-24 x log2 e ln 2) and two hardware functions of 1 ulp, and four more
products: below 60 x 2^-24 = 4e-6 of the value.  r = residual + scale x is one rounding of the sum."""
import numpy as np
import pytest
import torch

from oracle import block_oracle
from parity import to_np64

pytestmark = pytest.mark.gpu
F32_REL, BF16_REL = 4e-6, 2.0 ** -8 + 4e-6
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


@pytest.fixture(scope="module")
def ssd():
    from paper_2603_09555_amd import ssd as binding
    return binding


def close(got, ref, what, dtype):
    g = to_np64(got)
    rel = BF16_REL if dtype == torch.bfloat16 else F32_REL
    tiny = 1e-38   # below the smallest normal number roundings are absolute
    bad = ~(np.abs(g - ref) <= rel * np.abs(ref) + tiny)
    assert not bad.any(), "%s: %d of %d off, worst %.3e" % (what, bad.sum(), bad.size, np.abs((g - ref) / np.where(ref == 0, 1, ref)).max())


def draw(rows, width, io, seed, pad=0, scale=1.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn((rows, width + pad), generator=g) * scale).to(TYPES[io])


WIDTHS = [1, 2, 7, 8, 9, 63, 64, 65, 511, 512, 520, 1537, 2048, 2050, 5120, 8192, 8200, 20001]


@pytest.mark.parametrize("io", ["f32", "bf16"])
@pytest.mark.parametrize("norm_first", [False, True])
@pytest.mark.parametrize("width", WIDTHS)
def test_gated_norm_matches_oracle(ssd, width, norm_first, io):
    for rows, groups, pad in ((1, 1, 0), (5, 1, 3), (3, 2 if width % 2 == 0 else 1, 8), (2, width if width < 100 else 1, 1)):
        y, wide, w = draw(rows, width, io, 1), draw(rows, width, io, 2, pad), draw(1, width, "f32", 3)[0]
        z = wide[:, :width]
        print("gated", rows, width, groups, pad, io, flush=True)
        zd = wide.cuda()[:, pad:] if pad else wide.cuda()   # (a slice that begins at no multiple of 16 bytes)
        z = wide[:, pad:] if pad else z
        out = ssd.ssd_norm_gated(y.cuda(), zd, w.cuda(), groups=groups, norm_first=norm_first)
        torch.cuda.synchronize()
        close(out, block_oracle.norm_gated(y, z, w, 1e-5, groups, norm_first), "gated", y.dtype)


@pytest.mark.parametrize("io,stream", [("f32", "f32"), ("bf16", "f32"), ("bf16", "bf16")])
@pytest.mark.parametrize("width", WIDTHS)
def test_residual_norm_matches_oracle(ssd, width, io, stream):
    for rows, scale in ((1, 1.0), (5, 0.22), (33, -3.0)):
        x, res, w = draw(rows, width, io, 4), draw(rows, width, stream, 5, scale=3.0), draw(1, width, "f32", 6)[0]
        scale = float(np.float32(scale))
        print("residual", rows, width, io, stream, flush=True)
        out, r = ssd.ssd_norm_residual(res.cuda(), x.cuda(), w.cuda(), scale=scale)
        torch.cuda.synchronize()
        ref, r_ref = block_oracle.norm_residual(res, x, w, scale, 1e-5)
        close(r, r_ref, "stream", res.dtype)
        close(out, ref, "out", x.dtype)


@pytest.mark.parametrize("rows", [512, 513])
@pytest.mark.parametrize("width", [2050, 4096, 5117, 8192, 8200, 16384])
def test_norms_of_more_rows(ssd, width, rows):
    """Wide rows, on either side of the number from which a thread takes several pieces of them."""
    x, side, w = draw(rows, width, "bf16", 20), draw(rows, width, "bf16", 21), draw(1, width, "f32", 22)[0]
    print("norms", rows, width, flush=True)
    gated = ssd.ssd_norm_gated(x.cuda(), side.cuda(), w.cuda(), norm_first=True)
    out, r = ssd.ssd_norm_residual(side.cuda(), x.cuda(), w.cuda(), scale=0.5)
    torch.cuda.synchronize()
    some = slice(None, None, 37)
    close(gated[some], block_oracle.norm_gated(x[some], side[some], w, 1e-5, 1, True), "gated", x.dtype)
    ref, r_ref = block_oracle.norm_residual(side[some], x[some], w, 0.5, 1e-5)
    close(r[some], r_ref, "stream", side.dtype)
    close(out[some], ref, "out", x.dtype)


@pytest.mark.parametrize("stream", ["f32", "bf16"])
def test_first_block_has_no_residual(ssd, stream):
    x, w = draw(7, 300, "bf16", 7), draw(1, 300, "f32", 8)[0]
    given = torch.full((7, 300), float("nan"), dtype=TYPES[stream], device="cuda")
    out, r = ssd.ssd_norm_residual(None, x.cuda(), w.cuda(), scale=0.5, residual_out=given)
    torch.cuda.synchronize()
    ref, r_ref = block_oracle.norm_residual(None, x, w, 0.5, 1e-5)
    assert r is given
    close(r, r_ref, "stream", r.dtype)
    close(out, ref, "out", x.dtype)
    assert ssd.ssd_norm_residual(None, x.cuda(), w.cuda())[1].dtype == torch.float32


@pytest.mark.parametrize("width", [77, 5120, 20001])
def test_norms_in_place(ssd, width):
    """Outputs that are inputs get what separate outputs get."""
    y, z, w = draw(9, width, "bf16", 9).cuda(), draw(9, width, "bf16", 10).cuda(), draw(1, width, "f32", 11)[0].cuda()
    res = draw(9, width, "f32", 12).cuda()
    for norm_first in (False, True):
        ref = ssd.ssd_norm_gated(y, z, w, norm_first=norm_first)
        a = y.clone()
        assert ssd.ssd_norm_gated(a, z, w, norm_first=norm_first, out=a) is a and torch.equal(a, ref)
        b = z.clone()
        ssd.ssd_norm_gated(y, b, w, norm_first=norm_first, out=b)
        assert torch.equal(b, ref)
    out, r = ssd.ssd_norm_residual(res, y, w)
    a, s = y.clone(), res.clone()
    ssd.ssd_norm_residual(s, a, w, out=a, residual_out=s)
    assert torch.equal(a, out) and torch.equal(s, r)


def test_rows_of_zeros_and_extreme_gates(ssd):
    """eps keeps a row of zeros finite; gates far from zero neither overflow nor lose their sign."""
    y, z, w = torch.zeros(4, 96), torch.zeros(4, 96), torch.ones(96)
    y[1:] = 1.0
    z[1], z[2], z[3] = 200.0, -200.0, torch.linspace(-90, 90, 96)
    out = ssd.ssd_norm_gated(y.cuda(), z.cuda(), w.cuda()).cpu()
    assert torch.equal(out[0], torch.zeros(96)) and torch.isfinite(out).all()
    ref = block_oracle.norm_gated(y, z, w, 1e-5)
    assert np.abs(out.double().numpy() - ref).max() <= 2e-5 * np.abs(ref).max()
    assert ssd.ssd_norm_residual(None, y[:1].cuda(), w.cuda())[0].abs().max() == 0


def test_a_row_does_not_depend_on_the_others(ssd):
    """The same row alone and among many: the same bits."""
    y, z, w = draw(300, 1000, "bf16", 13).cuda(), draw(300, 1000, "bf16", 14).cuda(), draw(1, 1000, "f32", 15)[0].cuda()
    a = ssd.ssd_norm_gated(y, z, w)
    for i in (0, 137, 299):
        assert torch.equal(ssd.ssd_norm_gated(y[i:i + 1], z[i:i + 1], w), a[i:i + 1])


def test_rows_behind_four_gib(ssd):
    """Offsets of the last rows pass 32 bits."""
    rows, width = 70000, 32768
    y = torch.zeros((rows, width), dtype=torch.bfloat16, device="cuda")
    y[-3:] = draw(3, width, "bf16", 16).cuda()
    z = torch.zeros_like(y)
    z[-3:] = draw(3, width, "bf16", 17).cuda()
    w = draw(1, width, "f32", 18)[0].cuda()
    out = ssd.ssd_norm_gated(y, z, w, out=y)
    torch.cuda.synchronize()
    close(out[-3:], block_oracle.norm_gated(draw(3, width, "bf16", 16), draw(3, width, "bf16", 17), w.cpu(), 1e-5), "last rows", y.dtype)
    assert out[:-3].abs().max() == 0
