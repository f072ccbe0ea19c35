"""A row's bits do not depend on how many rows a call has, at the widths where the number of threads does."""
import pytest
import torch

from test_gpu_norm import draw, ssd  # noqa: F401

pytestmark = pytest.mark.gpu
WIDTHS = [2049, 2056, 4096, 5117, 5120, 6144, 6152, 8192, 8193, 12000, 16384, 16392, 20001]


@pytest.mark.parametrize("io", ["f32", "bf16"])
@pytest.mark.parametrize("width", WIDTHS)
def test_rows_alone_and_among_many(ssd, width, io):  # noqa: F811
    rows = 513
    y, z, w = draw(rows, width, io, 1).cuda(), draw(rows, width, io, 2).cuda(), draw(1, width, "f32", 3)[0].cuda()
    res = draw(rows, width, "f32", 4, scale=3.0).cuda()
    for first in (False, True):
        many = ssd.ssd_norm_gated(y, z, w, norm_first=first)
        for n in (1, 512):
            assert torch.equal(ssd.ssd_norm_gated(y[:n], z[:n], w, norm_first=first), many[:n]), n
        assert torch.equal(ssd.ssd_norm_gated(y[-1:], z[-1:], w, norm_first=first), many[-1:])
    out, r = ssd.ssd_norm_residual(res, y, w)
    for part in (slice(0, 1), slice(0, 512), slice(rows - 1, rows)):
        a, b = ssd.ssd_norm_residual(res[part], y[part], w)
        assert torch.equal(a, out[part]) and torch.equal(b, r[part])


def test_groups_alone_and_among_many(ssd):  # noqa: F811
    """Groups are units as rows are."""
    y, z, w = draw(70, 8 * 2560, "bf16", 5).cuda(), draw(70, 8 * 2560, "bf16", 6).cuda(), draw(1, 8 * 2560, "f32", 7)[0].cuda()
    many = ssd.ssd_norm_gated(y, z, w, groups=8)
    assert torch.equal(ssd.ssd_norm_gated(y[:1], z[:1], w, groups=8), many[:1])
