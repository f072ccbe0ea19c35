"""Sizes that 32 bits do not hold are refused by the binding and not cut to others, which the library might take."""
import pytest
import torch

from paper_2603_09555_amd import ssd

BIG = 2 ** 32 + 8


def meta(*shape, dtype=torch.bfloat16):
    return torch.empty(shape, dtype=dtype, device="meta")


def test_norms():
    f32 = torch.float32
    for call in (lambda: ssd.ssd_norm_gated(meta(1, BIG), meta(1, BIG), meta(BIG, dtype=f32)),
                 lambda: ssd.ssd_norm_gated(meta(1, 64), meta(1, 64), meta(64, dtype=f32), groups=2 ** 32 + 1),
                 lambda: ssd.ssd_norm_residual(None, meta(1, BIG), meta(BIG, dtype=f32))):
        with pytest.raises(ValueError, match="32 bits"):
            call()


def test_attention():
    cache, table = meta(5, 2, 16, 64), meta(3, 4, dtype=torch.int32)
    for args in ((BIG, 3, 4, cache, table), (3, BIG, 4, cache, table), (3, 3, BIG, cache, table), (3, 3, 4, meta(BIG, 2, 16, 64), table),
                 (3, 3, 4, meta(5, 2, BIG, 64), table), (3, 3, 4, cache, meta(3, BIG, dtype=torch.int32))):
        with pytest.raises(ValueError, match="32 bits"):
            ssd.make_attn_shape(*args)
    assert ssd.make_attn_shape(3, 3, 4, cache, table).npages == 5
