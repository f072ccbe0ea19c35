"""GPU parity of the operators on a paged key-value cache against the fp64 oracle, element by element.

Limits are those of the library's other kernels (parity.py): 1e-4 for fp32, 2e-2 for bf16, normalised and element-wise.  They
hold with room.  fp32: an exponent is a sum of at most 256 products, 256 x 2^-24 of sum |q k| scale (about 2 sqrt(headdim) here)
at worst, 1e-6 as random roundings add up.  bf16: a probability rounded to 8 significant bits is off by 2^-8 at most, with
random signs, so their sum by 2^-8 of y's own size, and y is rounded once, 2^-8: together below 1e-2.
Slots behind a sequence's end and pages of nobody hold NaN and infinities everywhere here."""
import numpy as np
import pytest
import torch

from oracle import block_oracle
from parity import TOL, assert_close, to_np64

pytestmark = pytest.mark.gpu
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


@pytest.fixture(scope="module")
def ssd():
    from paper_2603_09555_amd import ssd as binding
    return binding


def make(lengths, H, Hk, D, page, io, new=None, seed=0, spare=2, logits=2.0, more_pages=0):
    """A cache with the sequences' tokens in pages of no order, everything else poisoned."""
    g = torch.Generator().manual_seed(seed)
    t = TYPES[io]
    need = [-(-max(n, 0) // page) for n in lengths]
    npages = sum(need) + spare
    order = torch.randperm(npages, generator=g).to(torch.int32)
    table = torch.full((len(lengths), max(1, max(need)) + more_pages), -1, dtype=torch.int32)
    k, v = torch.randn((npages, Hk, page, D), generator=g).to(t), torch.randn((npages, Hk, page, D), generator=g).to(t)
    used = torch.zeros((npages, page), dtype=torch.bool)
    at = 0
    for b, n in enumerate(lengths):
        table[b, :need[b]] = order[at:at + need[b]]
        at += need[b]
        for p in range(need[b]):
            used[table[b, p], :min(page, n - p * page)] = True
    poison = torch.tensor([float("nan"), float("inf"), float("-inf")]).to(t)
    hole = (~used).nonzero()
    for i, (p, s) in enumerate(hole.tolist()):
        k[p, :, s] = poison[i % 3]
        v[p, :, s] = poison[(i + 1) % 3]
    new = [1] * len(lengths) if new is None else new
    cu = torch.tensor([0] + list(np.cumsum(new)), dtype=torch.int32)
    q = (logits * torch.randn((int(cu[-1]), H, D), generator=g)).to(t)
    return dict(q=q, k=k, v=v, table=table, lens=torch.tensor(lengths, dtype=torch.int32), cu=cu)


def dev(s):
    return {n: t.cuda() for n, t in s.items()}


def run_step(ssd, s, **kw):
    d = dev(s)
    y = ssd.ssd_attn_step(d["q"], d["k"], d["v"], d["table"], d["lens"], **kw)
    torch.cuda.synchronize()
    return y


def run_prefill(ssd, s, **kw):
    d = dev(s)
    y = ssd.ssd_attn_prefill(d["q"], d["k"], d["v"], d["table"], d["lens"], d["cu"], **kw)
    torch.cuda.synchronize()
    return y


HEADS = [  # H, Hk, D, page
    (1, 1, 64, 16), (4, 4, 128, 16), (32, 8, 128, 16), (5, 1, 64, 64), (14, 2, 80, 32), (16, 1, 128, 1), (40, 2, 64, 128),
    (2, 2, 256, 16), (8, 2, 8, 4), (6, 3, 24, 8), (9, 3, 200, 2), (33, 1, 112, 16), (4, 1, 96, 4096),
]
LENGTHS = [[1], [0], [2, 0, 31], [32, 33, 63, 64, 65], [127, 128, 129, 500], [1000, 1, 3, 2049]]


@pytest.mark.parametrize("io", ["f32", "bf16"])
@pytest.mark.parametrize("heads", HEADS, ids=lambda h: "x".join(map(str, h)))
def test_step_matches_oracle(ssd, heads, io):
    for i, lengths in enumerate(LENGTHS + LENGTHS):
        # (a wide page table: sequences might be long, and work is dealt to the workgroups by length)
        s = make(lengths, *heads, io, seed=i, more_pages=0 if i < len(LENGTHS) else -(-600000 // heads[2] // heads[3]))
        for window in (0, 1, 40):
            print("step", heads, io, lengths, window, s["table"].shape[1], flush=True)
            y = run_step(ssd, s, window=window)
            assert_close(y, block_oracle.attention(s["q"], s["k"], s["v"], s["table"], s["lens"], window=window), TOL[io], "step")


@pytest.mark.parametrize("batch", [64, 65, 257, 700])
def test_step_many_sequences_dealt(ssd, batch):
    """More sequences than a wave, or a workgroup, has lanes, many of them empty; the table is wide, so that work is dealt."""
    lengths = np.random.default_rng(batch).integers(0, 300, batch)
    lengths[::3] = 0
    lengths[-1] = 0
    s = make([int(n) for n in lengths], 6, 2, 64, 16, "bf16", seed=batch, more_pages=700)
    for window in (0, 100):
        print("step", batch, window, flush=True)
        y = run_step(ssd, s, window=window)
        assert_close(y, block_oracle.attention(s["q"], s["k"], s["v"], s["table"], s["lens"], window=window), TOL["bf16"], "step")


@pytest.mark.parametrize("io", ["f32", "bf16"])
@pytest.mark.parametrize("heads", [(4, 2, 64, 16), (3, 1, 128, 1), (2, 1, 256, 64), (20, 1, 72, 8)], ids=lambda h: "x".join(map(str, h)))
def test_step_many_short_sequences(ssd, heads, io):
    """More sequences and key heads than CUs, none of them long."""
    lengths = np.random.default_rng(7).integers(0, 200, 300)
    lengths[::7] = 0
    s = make([int(n) for n in lengths], *heads, io, seed=60)
    for window in (0, 33):
        print("step", heads, io, window, flush=True)
        y = run_step(ssd, s, window=window)
        assert_close(y, block_oracle.attention(s["q"], s["k"], s["v"], s["table"], s["lens"], window=window), TOL[io], "step")


@pytest.mark.parametrize("io", ["f32", "bf16"])
@pytest.mark.parametrize("headdim", [64, 128, 256])
@pytest.mark.parametrize("batch", [3, 150])
def test_step_on_large_caches(ssd, batch, headdim, io):
    """Caches of more than the last-level cache holds, of which little is used: work dealt, and a unit to a workgroup."""
    lengths = np.random.default_rng(8).integers(1, 300, batch)
    s = make([int(n) for n in lengths], 4, 2, headdim, 16, io, seed=61, more_pages=-(-600000 // headdim // 16) if batch == 3 else 0)
    d = dev(s)
    pages = 360 * 1024 * 1024 // (2 * 2 * 16 * headdim * (2 if io == "bf16" else 4))
    k, v = (torch.full((pages, 2, 16, headdim), float("nan"), dtype=t.dtype, device="cuda") for t in (d["k"], d["v"]))
    k[-d["k"].shape[0]:], v[-d["v"].shape[0]:] = d["k"], d["v"]
    table = torch.where(d["table"] < 0, d["table"], d["table"] + pages - d["k"].shape[0])
    print("step", batch, headdim, io, pages, flush=True)
    y = ssd.ssd_attn_step(d["q"], k, v, table, d["lens"])
    torch.cuda.synchronize()
    assert_close(y, block_oracle.attention(s["q"], s["k"], s["v"], s["table"], s["lens"]), TOL[io], "step")


PIECES = [  # new tokens, cached tokens
    ([1], [0]), ([5], [0]), ([0, 3, 0, 0, 70, 1], [9, 0, 0, 5, 130, 64]), ([64, 65, 63], [0, 64, 1]), ([260], [0]), ([7, 129], [1000, 513]),
]


@pytest.mark.parametrize("io", ["f32", "bf16"])
@pytest.mark.parametrize("heads", HEADS, ids=lambda h: "x".join(map(str, h)))
def test_prefill_matches_oracle(ssd, heads, io):
    for i, (new, prior) in enumerate(PIECES):
        s = make([a + b for a, b in zip(new, prior)], *heads, io, new=new, seed=10 + i)
        for window in (0, 1, 50):
            print("prefill", heads, io, new, prior, window, flush=True)
            y = run_prefill(ssd, s, window=window)
            ref = block_oracle.attention(s["q"], s["k"], s["v"], s["table"], s["lens"], s["cu"], window=window)
            assert_close(y, ref, TOL[io], "prefill")


@pytest.mark.parametrize("heads", [(6, 2, 64, 16), (4, 2, 128, 16), (2, 1, 256, 16)], ids=lambda h: "x".join(map(str, h)))
def test_prefill_f32_is_exact_over_the_range(ssd, heads):
    """The values' parts lose nothing: a power of two goes through to the results bit by bit.  What is infinite and seen shows."""
    s = make([300, 70], *heads, "f32", new=[130, 70], seed=40)
    y = run_prefill(ssd, s)
    v = s["v"]
    for power in (100, -60):
        s["v"] = v * 2.0 ** power
        assert torch.equal(run_prefill(ssd, s), y * 2.0 ** power), power
    s["v"] = v.clone()
    s["v"][s["table"][0, 0], 0, 0, 3] = float("inf")  # the first token of the first sequence, which all of its rows see
    y = run_prefill(ssd, s)
    groups = heads[0] // heads[1]
    assert not torch.isfinite(y[:130, :groups, 3]).any()
    assert torch.isfinite(y[130:]).all() and torch.isfinite(y[:130, groups:]).all() and torch.isfinite(y[:130, :, :3]).all()


@pytest.mark.parametrize("io", ["f32", "bf16"])
@pytest.mark.parametrize("batch", [2, 64, 65, 150])
def test_prefill_many_sequences(ssd, batch, io):
    """Pieces of few and of many tokens, some of them behind a long cache, whose units are shared, and some with nothing new."""
    rng = np.random.default_rng(batch)
    new, prior = rng.integers(0, 40, batch), rng.integers(0, 60, batch)
    new[::3] = 0
    new[-2], prior[-2] = 150, 2500
    new[0], prior[0] = 3, 1700
    s = make([int(n) for n in new + prior], 3, 1, 64, 16, io, new=[int(n) for n in new], seed=batch)
    for window in (0, 700):
        print("prefill", batch, io, window, flush=True)
        y = run_prefill(ssd, s, window=window)
        ref = block_oracle.attention(s["q"], s["k"], s["v"], s["table"], s["lens"], s["cu"], window=window)
        assert_close(y, ref, TOL[io], "prefill")


@pytest.mark.parametrize("io", ["f32", "bf16"])
@pytest.mark.parametrize("batch", [65, 200, 4200])
def test_prefill_many_units(ssd, batch, io):
    """Units enough for every CU several times over: sequences are searched for, in steps of 64."""
    rng = np.random.default_rng(batch)
    new, prior = rng.integers(0, 9, batch), rng.integers(0, 20, batch)
    new[rng.integers(0, batch, batch // 4)] = 0
    new[-1] = 0
    new[batch // 2] = 150
    s = make([int(n) for n in new + prior], 24, 12, 16, 8, io, new=[int(n) for n in new], seed=batch)
    print("prefill", batch, io, flush=True)
    y = run_prefill(ssd, s)
    assert_close(y, block_oracle.attention(s["q"], s["k"], s["v"], s["table"], s["lens"], s["cu"]), TOL[io], "prefill")


@pytest.mark.parametrize("io", ["f32", "bf16"])
def test_prefill_late_pieces_of_many_heads(ssd, io):
    """Pieces with enough to do for every CU that the number of rounds decides how units are shared."""
    new, prior = [40, 30, 23, 0, 40], [19000, 18500, 17000, 100, 18990]
    s = make([a + b for a, b in zip(new, prior)], 48, 24, 16, 32, io, new=new, seed=70)
    print("prefill late", io, flush=True)
    y = run_prefill(ssd, s)
    some = slice(None, None, 11)
    q, cu = s["q"], s["cu"]
    ref = block_oracle.attention(q, s["k"], s["v"], s["table"], s["lens"], cu)
    assert_close(y[some], ref[some], TOL[io], "prefill")


def test_prefill_overlapping_boundaries_stay_inside(ssd):
    """Boundaries that count tokens many times over: results are anything, what surrounds y and the caches stays as it was."""
    s = make([3000] * 40, 4, 1, 64, 16, "bf16", new=[20] * 40, seed=50)
    s["cu"] = torch.tensor([0, 800] * 20 + [0], dtype=torch.int32)
    d = dev(s)
    k, v = d["k"].clone(), d["v"].clone()
    room = torch.full((802, 4, 64), 7.0, dtype=torch.bfloat16, device="cuda")
    ssd.ssd_attn_prefill(d["q"], d["k"], d["v"], d["table"], d["lens"], d["cu"], y=room[1:801])
    torch.cuda.synchronize()
    assert bool((room[0] == 7).all()) and bool((room[801] == 7).all())
    assert torch.equal(d["k"].view(torch.int16), k.view(torch.int16)) and torch.equal(d["v"].view(torch.int16), v.view(torch.int16))


@pytest.mark.parametrize("io", ["f32", "bf16"])
def test_long_step_and_prefill(ssd, io):
    """Enough work for every workgroup, split and joined: a long sequence among short ones, and a late piece of a prompt."""
    s = make([20011, 17, 900], 10, 2, 128, 16, io, seed=30)
    for window in (0, 3000):
        y = run_step(ssd, s, window=window)
        assert_close(y, block_oracle.attention(s["q"], s["k"], s["v"], s["table"], s["lens"], window=window), TOL[io], "step")
    s = make([9000, 700], 4, 2, 128, 64, io, new=[200, 700], seed=31)
    for window in (0, 1025):
        y = run_prefill(ssd, s, window=window)
        ref = block_oracle.attention(s["q"], s["k"], s["v"], s["table"], s["lens"], s["cu"], window=window)
        assert_close(y, ref, TOL[io], "prefill")


def test_many_sequences(ssd):
    """More sequences than a wave, and than a workgroup, has lanes; most are short, some are empty."""
    lengths = [(i * 7) % 90 for i in range(700)]
    s = make(lengths, 2, 1, 64, 16, "bf16", seed=32)
    ref = block_oracle.attention(s["q"], s["k"], s["v"], s["table"], s["lens"])
    assert_close(run_step(ssd, s), ref, TOL["bf16"], "step")
    s["table"] = torch.cat((s["table"], torch.full((700, 1000), -1, dtype=torch.int32)), dim=1)
    assert_close(run_step(ssd, s), ref, TOL["bf16"], "step, dealt")
    new = [min(n, (i * 5) % 4) for i, n in enumerate(lengths)]
    s = make(lengths, 2, 1, 64, 16, "bf16", new=new, seed=33)
    ref = block_oracle.attention(s["q"], s["k"], s["v"], s["table"], s["lens"], s["cu"])
    assert_close(run_prefill(ssd, s), ref, TOL["bf16"], "prefill")


@pytest.mark.parametrize("io", ["f32", "bf16"])
def test_steep_logits_and_given_scale(ssd, io):
    """Logits up to some hundreds: the softmax is a choice, and its running maximum moves by much."""
    s = make([700, 70], 4, 2, 64, 16, io, new=[300, 70], seed=34, logits=40.0)
    # fp32 logits of size 400 carry 400 x 2^-24 x a few: limits of the exponent's error, not of the kernel's steps
    ref = block_oracle.attention(s["q"], s["k"], s["v"], s["table"], s["lens"], s["cu"], scale=0.3)
    assert_close(run_prefill(ssd, s, scale=0.3), ref, 10 * TOL["f32"] if io == "f32" else TOL[io], "prefill")
    s = make([700, 70], 4, 2, 64, 16, io, seed=35, logits=40.0)
    ref = block_oracle.attention(s["q"], s["k"], s["v"], s["table"], s["lens"], scale=0.3)
    assert_close(run_step(ssd, s, scale=0.3), ref, 10 * TOL["f32"] if io == "f32" else TOL[io], "step")


@pytest.mark.parametrize("io", ["f32", "bf16"])
def test_odd_device_arrays(ssd, io):
    """Lengths beyond the table or below zero, pages that are not in the cache, boundaries out of order or beyond the tokens, more
    new tokens than a sequence has: what ssd.h says of each."""
    s = make([90, 70, 33, 200], 4, 2, 64, 16, io, new=[10, 40, 20, 30], seed=36)
    s["lens"] = torch.tensor([90, -5, 12, 10000], dtype=torch.int32)   # (the last is cut to its row of the table, 208)
    npages = s["k"].shape[0]
    s["table"][0, 1], s["table"][0, 3] = -7, npages     # two pages in the middle that nobody has
    s["table"][3, 12] = npages + 100000                 # and the last one
    given = torch.full(s["q"].shape, 7.0, dtype=s["q"].dtype)
    for cu in ([0, 10, 50, 70, 100], [5, 10, 10, 40, 90], [0, 10, 50, 70, 250], [-3, 20, 20, 20, 100], [0, 0, 0, 0, 0]):
        s["cu"] = torch.tensor(cu, dtype=torch.int32)
        for window in (0, 20):
            y = given.cuda()
            run_prefill(ssd, s, window=window, y=y)
            ref = block_oracle.attention(s["q"], s["k"], s["v"], s["table"], s["lens"], s["cu"], window=window, y=given)
            assert_close(y, ref, TOL[io], "prefill %s" % cu)
    s["q"] = s["q"][:4].contiguous()
    assert_close(run_step(ssd, s), block_oracle.attention(s["q"], s["k"], s["v"], s["table"], s["lens"]), TOL[io], "step")
    # out of order: nothing faults, and a sequence between boundaries in order is right
    s = make([90, 70, 33], 4, 2, 64, 16, io, new=[10, 40, 20], seed=37)
    s["cu"] = torch.tensor([0, 10, 5, 70], dtype=torch.int32)
    run_prefill(ssd, s)
    d = dev(s)
    ssd.ssd_attn_append(d["q"], torch.zeros(70, 2, 64, device="cuda").to(TYPES[io]), torch.zeros(70, 2, 64, device="cuda").to(TYPES[io]), d["k"], d["v"],
                        d["table"], d["lens"], d["cu"])
    torch.cuda.synchronize()


def rope_table(positions, rotary):
    half = rotary // 2
    a = np.arange(positions)[:, None] * 10000.0 ** (-np.arange(half) / max(half, 1))[None]
    return torch.tensor(np.cos(a), dtype=torch.float32), torch.tensor(np.sin(a), dtype=torch.float32)


APPENDS = [  # H, Hk, D, page, rotary, interleaved
    (32, 8, 128, 16, 128, False), (4, 2, 64, 32, 64, True), (5, 1, 80, 16, 32, False), (4, 4, 64, 8, 20, False), (3, 3, 24, 16, 6, True),
    (2, 1, 256, 64, 0, False), (2, 2, 8, 1, 8, False), (6, 2, 200, 4, 200, False), (1, 1, 72, 16, 36, True),
]


@pytest.mark.parametrize("io", ["f32", "bf16"])
@pytest.mark.parametrize("case", APPENDS, ids=lambda c: "x".join(map(str, c)))
def test_append_matches_oracle(ssd, case, io):
    """Rotated values are one fp32 product and one fused sum: 2 x 2^-24 of |a| + |b|, and the rounding to io."""
    H, Hk, D, page, rotary, interleaved = case
    for i, (new, prior) in enumerate((([1, 1, 1], [0, 40, 15]), ([17, 0, 33, 1], [3, 20, 0, 64]))):
        s = make([a + b for a, b in zip(new, prior)], H, Hk, D, page, io, new=new, seed=40 + i)
        tokens = int(s["cu"][-1])
        g = torch.Generator().manual_seed(50 + i)
        qkv = torch.randn((tokens, (H + 2 * Hk) * D + 8), generator=g).to(TYPES[io])
        rope = rope_table(s["table"].shape[1] * page, rotary) if rotary else None
        parts = [t.unflatten(1, (-1, D)) for t in qkv[:, :(H + 2 * Hk) * D].split((H * D, Hk * D, Hk * D), dim=1)]
        w = qkv.cuda()[:, :(H + 2 * Hk) * D].split((H * D, Hk * D, Hk * D), dim=1)
        d = dev(s)
        print("append", case, io, new, flush=True)
        q_out = ssd.ssd_attn_append(*[t.unflatten(1, (-1, D)) for t in w], d["k"], d["v"], d["table"], d["lens"],
                                    None if i == 0 else d["cu"], rope=None if rope is None else [t.cuda() for t in rope], interleaved=interleaved)
        torch.cuda.synchronize()
        ref = block_oracle.append(*parts, s["k"], s["v"], s["table"], s["lens"], None if i == 0 else s["cu"], rope, interleaved)
        size = np.abs(np.concatenate([to_np64(t).reshape(-1) for t in parts])).max()
        rel = 2.0 ** -8 if io == "bf16" else 2.0 ** -24
        for got, want, what in zip((q_out, d["k"], d["v"]), ref, ("q", "k", "v")):
            g64 = got.double().cpu().numpy()
            same = (g64 == want) | (np.isnan(g64) & np.isnan(want))
            with np.errstate(invalid="ignore"):
                near = np.abs(g64 - want) <= rel * np.abs(want) + 4 * 2.0 ** -24 * size
            assert (same | near).all(), what
        assert torch.equal(d["v"].cpu().nan_to_num(nan=3.0), torch.tensor(ref[2]).to(TYPES[io]).nan_to_num(nan=3.0)), "values are copied"


def test_append_without_queries_and_odd_tokens(ssd):
    """Keys and values alone; tokens in front of a sequence's beginning, of absent pages and of nobody leave no trace."""
    s = make([20, 3, 40], 2, 2, 64, 16, "bf16", new=[4, 6, 5], seed=60)
    s["table"][2, 2] = -1
    s["cu"][3] = 13
    g = torch.Generator().manual_seed(61)
    q, k, v = (torch.randn((15, 2, 64), generator=g).bfloat16() for _ in range(3))
    d = dev(s)
    assert ssd.ssd_attn_append(None, k.cuda(), v.cuda(), d["k"], d["v"], d["table"], d["lens"], d["cu"]) is None
    given = torch.full((15, 2, 64), 5.0, dtype=torch.bfloat16)
    _, k_ref, v_ref = block_oracle.append(None, k, v, s["k"], s["v"], s["table"], s["lens"], s["cu"])
    assert np.array_equal(d["k"].double().cpu().numpy(), k_ref, equal_nan=True) and np.array_equal(d["v"].double().cpu().numpy(), v_ref, equal_nan=True)
    q_out = ssd.ssd_attn_append(q.cuda(), k.cuda(), v.cuda(), d["k"], d["v"], d["table"], d["lens"], d["cu"], q_out=given.cuda())
    q_ref, _, _ = block_oracle.append(q, k, v, s["k"], s["v"], s["table"], s["lens"], s["cu"], q_out=given)
    assert np.array_equal(q_out.double().cpu().numpy(), q_ref)


def test_pages_behind_four_gib(ssd):
    """A cache of 9 GiB (keys and values): the offsets of the last pages pass 32 bits, in bytes and in values."""
    npages, Hk, page, D = 70000, 4, 64, 128
    k = torch.zeros((npages, Hk, page, D), dtype=torch.bfloat16, device="cuda")
    v = torch.zeros_like(k)
    g = torch.Generator().manual_seed(62)
    table = torch.tensor([[npages - 1, 3, npages - 2], [npages - 3, 69000, 0]], dtype=torch.int32)
    lens = torch.tensor([150, 100], dtype=torch.int32)
    cu = torch.tensor([0, 150, 250], dtype=torch.int32)
    q, kn, vn = (torch.randn((250, h, D), generator=g).bfloat16() for h in (8, Hk, Hk))
    d = [t.cuda() for t in (q, kn, vn)]
    ssd.ssd_attn_append(None, d[1], d[2], k, v, table.cuda(), lens.cuda(), cu.cuda())
    y = ssd.ssd_attn_prefill(d[0], k, v, table.cuda(), lens.cuda(), cu.cuda())
    ys = ssd.ssd_attn_step(d[0][[149, 249]].contiguous(), k, v, table.cuda(), lens.cuda())
    torch.cuda.synchronize()
    # the oracle's cache holds the pages in use alone
    small = {int(p): i for i, p in enumerate(table.flatten())}
    kc, vc = torch.zeros(6, Hk, page, D, dtype=torch.bfloat16), torch.zeros(6, Hk, page, D, dtype=torch.bfloat16)
    t2 = torch.tensor([[small[int(p)] for p in row] for row in table], dtype=torch.int32)
    _, kc, vc = block_oracle.append(None, kn, vn, kc, vc, t2, lens, cu)
    assert np.array_equal(k[table.flatten().long()].double().cpu().numpy(), kc)
    ref = block_oracle.attention(q, kc, vc, t2, lens, cu)
    assert_close(y, ref, TOL["bf16"], "prefill")
    assert_close(ys, ref[[149, 249]], TOL["bf16"], "step")
    assert k[1].abs().max() == 0 and k[npages // 2].abs().max() == 0


@pytest.mark.parametrize("io", ["f32", "bf16"])
def test_runs_repeat_bit_for_bit_and_on_other_streams(ssd, io):
    s = make([3000, 10, 513], 8, 2, 128, 16, io, new=[40, 10, 200], seed=63)
    d = dev(s)
    q1 = d["q"][:3].contiguous()
    args = (d["k"], d["v"], d["table"], d["lens"])
    y, ys = ssd.ssd_attn_prefill(d["q"], *args, d["cu"]), ssd.ssd_attn_step(q1, *args)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        for _ in range(3):
            assert torch.equal(ssd.ssd_attn_prefill(d["q"], *args, d["cu"]), y) and torch.equal(ssd.ssd_attn_step(q1, *args), ys)
    side.synchronize()


def test_a_captured_step_follows_growing_sequences(ssd):
    """Append and step captured once: every replay appends a token, sees it, and equals the eager calls bit for bit."""
    H, Hk, D, page = 8, 2, 128, 16
    lengths = [37, 1, 500]
    s = make([n + 20 for n in lengths], H, Hk, D, page, "bf16", seed=64)
    d = dev(s)
    lens = torch.tensor(lengths, dtype=torch.int32, device="cuda")
    g = torch.Generator(device="cuda").manual_seed(65)
    q, k, v = (torch.randn((3, h, D), generator=g, device="cuda").bfloat16() for h in (H, Hk, Hk))
    rope = [t.cuda() for t in rope_table(s["table"].shape[1] * page, D)]
    q_out, y = torch.empty_like(q), torch.empty_like(q)
    ws = torch.empty(max(256, ssd.attn_step_workspace_bytes(ssd.make_attn_shape(3, 3, H, d["k"], d["table"]))), dtype=torch.uint8, device="cuda")

    def step(k_cache, v_cache, out, rotated):
        ssd.ssd_attn_append(q, k, v, k_cache, v_cache, d["table"], lens, rope=rope, q_out=rotated)
        ssd.ssd_attn_step(rotated, k_cache, v_cache, d["table"], lens, y=out, workspace=ws)

    step(d["k"], d["v"], y, q_out)
    torch.cuda.synchronize()
    ek, ev = d["k"].clone(), d["v"].clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=torch.cuda.Stream()):
        step(d["k"], d["v"], y, q_out)
    for rep in range(6):
        lens += 3
        for t in (q, k, v):
            t.copy_(torch.randn(t.shape, generator=g, device="cuda").bfloat16())
        graph.replay()
        ey, eq = torch.empty_like(q), torch.empty_like(q)
        step(ek, ev, ey, eq)
        torch.cuda.synchronize()
        assert torch.equal(y, ey) and torch.equal(q_out, eq), rep
        assert torch.equal(d["k"].nan_to_num(), ek.nan_to_num()) and torch.equal(d["v"].nan_to_num(), ev.nan_to_num())
