"""The append with normed heads where a lane takes several heads: 3, 5 and 8 of them (two are on their way at a time), units of heads
that are not full among them.  Limits are derived in test_gpu_append_norm.py."""
import pytest

from test_gpu_append_norm import compare, make

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ssd():
    from paper_2603_09555_amd import ssd as binding
    return binding


# Heads a lane are a 4096th of the waves that one head a lane would take, at most 8.  Those are, for a token, the heads over the heads
# that 64 lanes hold, rounded up, of queries and twice of keys: 8 heads of 64 in bf16, 4 in fp32, 4 of 80 in bf16.
@pytest.mark.parametrize("tokens,H,Hk,D,rotary,io,interleaved", [
    (1800, 40, 8, 64, 64, "bf16", False),    # 5 + 2 waves, 12600 / 4096 = 3: 24 and 16 queries of 24, 8 keys of 24
    (6000, 40, 8, 64, 64, "bf16", False),    # 42000: 8: 40 queries of 64
    (2300, 36, 9, 64, 32, "bf16", True),     # 5 + 4, 20700: 5: 36 of 40, 9 of 40
    (900, 40, 8, 64, 64, "f32", False),      # 10 + 4, 12600: 3: 12, 12, 12 and 4 queries of 12
    (2400, 40, 8, 64, 64, "f32", True),      # 33600: 8: 32 and 8 queries of 32
    (1500, 40, 8, 80, 40, "bf16", False),    # 10 + 4, 21000: 5; rotated halves of 20, so that pieces hold values of both
    (2400, 38, 2, 80, 40, "bf16", False),    # 10 + 2, 28800: 7: 28 and 10 queries of 28
])
def test_several_heads_a_lane(ssd, tokens, H, Hk, D, rotary, io, interleaved):
    print("append", tokens, H, Hk, D, rotary, io, interleaved, flush=True)
    new = [tokens - 500, 0, 490, 3]
    compare(ssd, make(new, [3, 1, 30, 0], H, Hk, D, 16, rotary, io, seed=H + D, gaps=(2, 5)), io, interleaved)
