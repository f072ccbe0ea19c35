"""Norms of more rows, and of more groups, than one launch has threads for.  Limits as in test_gpu_norm.py."""
import pytest
import torch

from oracle import block_oracle
from test_gpu_norm import close, draw, ssd  # noqa: F401

pytestmark = pytest.mark.gpu


def places(n):
    """Both ends, and either side of the multiples of 2^27 and 2^21 units, where launches may begin."""
    at = [0, n - 1] + [k << 27 for k in range(1, 1 + (n >> 27))] + [1 << 21, 5 << 21, 1 << 23]
    return torch.tensor(sorted({min(max(i + d, 0), n - 1) for i in at for d in range(-40, 41)}))


def test_groups_of_one_value(ssd):  # noqa: F811
    rows, width = 65537, 4096          # 2^28 + 4096 groups of a value
    g = torch.Generator(device="cuda").manual_seed(1)
    y = torch.randn((rows, width), generator=g, device="cuda", dtype=torch.float32).bfloat16()
    z = torch.randn((rows, width), generator=g, device="cuda", dtype=torch.float32).bfloat16()
    w = draw(1, width, "f32", 2)[0]
    out = torch.full_like(y, float("nan"))
    print("gated", rows, width, flush=True)
    ssd.ssd_norm_gated(y, z, w.cuda(), groups=width, out=out)
    torch.cuda.synchronize()
    assert bool(torch.isfinite(out).all())
    some = torch.unique(places(rows * width) // width)
    close(out.cpu()[some], block_oracle.norm_gated(y.cpu()[some], z.cpu()[some], w, 1e-5, width), "gated", y.dtype)


@pytest.mark.parametrize("rows,width", [((1 << 28) + 5, 1), ((1 << 24) + 3, 520)])
def test_rows(ssd, rows, width):  # noqa: F811
    g = torch.Generator(device="cuda").manual_seed(3)
    x = torch.empty((rows, width), device="cuda", dtype=torch.bfloat16).normal_(generator=g)
    w = draw(1, width, "f32", 4)[0] + 2.0
    out, r = (torch.full_like(x, float("nan")) for _ in range(2))
    print("residual", rows, width, flush=True)
    ssd.ssd_norm_residual(None, x, w.cuda(), scale=0.5, out=out, residual_out=r)
    torch.cuda.synchronize()
    for part in torch.split(out, 1 << 22):
        assert bool(torch.isfinite(part).all())
    some = places(rows).cuda()
    ref, r_ref = block_oracle.norm_residual(None, x[some].cpu(), w, 0.5, 1e-5)
    close(out[some], ref, "out", x.dtype)
    close(r[some], r_ref, "stream", x.dtype)
