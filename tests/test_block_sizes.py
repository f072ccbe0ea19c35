"""Calls of more workgroups of 256 threads than a launch takes (less than 2^32 threads) are refused as shapes, not by the launch;
the largest that fit are not.  Nothing here reaches a launch."""
import ctypes

import pytest

from paper_2603_09555_amd import ssd
from test_block_abi import FAKE, shape

MOST = (1 << 24) - 1     # workgroups


@pytest.mark.parametrize("kw,workgroups", [
    (dict(batch=1 << 21, nheads=8, nkvheads=8), 1 << 24),
    (dict(batch=(1 << 21) - 1, nheads=8, nkvheads=8), (1 << 24) - 8),
    (dict(batch=1 << 20, nheads=34, nkvheads=2), 3 << 21),                      # three tiles of 16 heads
    (dict(batch=1 << 21, nheads=8, nkvheads=8, max_pages=1 << 16), 1 << 24),    # (long rows: the joining launch)
    (dict(batch=1 << 20, nheads=16, nkvheads=8, max_pages=1 << 16), 1 << 24),   # which cuts a unit of two heads
    (dict(batch=1 << 20, nheads=8, nkvheads=8, max_pages=1 << 16), 1 << 23)])
def test_step(kw, workgroups):
    s, fits = shape(**kw), workgroups <= MOST
    assert (ssd.attn_step_workspace_bytes(s) > 0) == fits
    st = ssd.raw().ssd_attn_step(ctypes.byref(s), FAKE, FAKE, FAKE, FAKE, FAKE, ctypes.c_float(0.1), None, FAKE, ctypes.c_size_t(1 << 50), None)
    assert st == (-1 if fits else -2)      # (what fits is looked at further: y is missing)


@pytest.mark.parametrize("kw,fits", [
    (dict(tokens=1 << 24, nheads=120, nkvheads=120, batch=8738), True),     # 15728640 + 120 x 8738: 2^24 - 16
    (dict(tokens=1 << 24, nheads=120, nkvheads=120, batch=8739), False)])
def test_prefill(kw, fits):
    s = shape(**kw)
    assert (ssd.attn_prefill_workspace_bytes(s) > 0) == fits
    st = ssd.raw().ssd_attn_prefill(ctypes.byref(s), FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, ctypes.c_float(0.1), None, FAKE, ctypes.c_size_t(1 << 50), None)
    assert st == (-1 if fits else -2)


@pytest.mark.parametrize("tokens,fits", [((1 << 26) - 4, True), (1 << 26, False)])   # four tokens a workgroup
def test_append(tokens, fits):
    s, rope = shape(tokens=tokens), ssd.ssd_rope(None, None, 0, 0, 0)
    i64 = ctypes.c_int64
    st = ssd.raw().ssd_attn_append(ctypes.byref(s), ctypes.byref(rope), FAKE, FAKE, FAKE, FAKE, i64(512), FAKE, i64(128), FAKE, i64(128), FAKE, None,
                                   FAKE, None)
    assert st == (-1 if fits else -2)
