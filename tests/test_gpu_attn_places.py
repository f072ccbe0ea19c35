"""New tokens that have no place in their sequence's row of the page table: in front of its beginning, or behind its last page.
They are not appended, see nothing (y = 0) and leave the others as they are without them.  Limits as in test_gpu_attn.py."""
import numpy as np
import pytest
import torch

from oracle import block_oracle
from parity import TOL, assert_close
from test_gpu_attn import TYPES, dev, make, rope_table, run_prefill, run_step, ssd  # noqa: F401

pytestmark = pytest.mark.gpu
HEADS = [(4, 2, 64, 16), (3, 1, 128, 1), (8, 1, 256, 32), (6, 3, 24, 8), (40, 2, 128, 16)]


def grown(heads, io, over, new, seed=0):
    """Sequences that fill their rows of the table, and whose lengths count ``over`` tokens more (None: a sequence that fits)."""
    H, Hk, D, page = heads
    full = 8 * 32 if page > 1 else 96
    lengths = [full if o is not None else full - 37 for o in over]
    s = make(lengths, H, Hk, D, page, io, new=new, seed=seed)
    s["lens"] += torch.tensor([o or 0 for o in over], dtype=torch.int32)
    return s, full


def expected(s, full, window):
    """Row by row: a token in front of the row's end as in a sequence that ends with it, the others nothing."""
    ref, cu = np.zeros(tuple(s["q"].shape)), s["cu"].tolist()
    for b in range(len(cu) - 1):
        n = cu[b + 1] - cu[b]
        kept = min(n, max(0, n - (int(s["lens"][b]) - full)))
        if kept == 0:
            continue
        rows = slice(cu[b], cu[b] + kept)
        ref[rows] = block_oracle.attention(s["q"][rows], s["k"], s["v"], s["table"][b:b + 1], s["lens"][b:b + 1] - (n - kept),
                                           torch.tensor([0, kept]), window=window)
    return ref


@pytest.mark.parametrize("io", ["f32", "bf16"])
@pytest.mark.parametrize("heads", HEADS, ids=lambda h: "x".join(map(str, h)))
def test_attention_behind_the_last_page(ssd, heads, io):  # noqa: F811
    for i, (over, new) in enumerate((([3, None], [5, 4]), ([None, 1, 70], [90, 64, 70]), ([2 ** 31 - 1 - 256], [40]), ([200, 0], [256, 10]))):
        if heads[3] == 1:
            new = [min(n, 59) for n in new]
        s, full = grown(heads, io, over, new, seed=i)
        for window in (0, 20):
            print("prefill", heads, io, over, new, window, flush=True)
            y = run_prefill(ssd, s, window=window)
            assert_close(y, expected(s, full, window), TOL[io], "prefill")
        s["q"] = s["q"][:len(over)].contiguous()
        for more in (0, 9000):    # (a wide table: the row is longer, and nobody is behind it)
            s["table"] = torch.nn.functional.pad(s["table"], (0, more), value=-1)
            y = run_step(ssd, s).cpu()
            for b in range(len(over)):
                behind = int(s["lens"][b]) > s["table"].shape[1] * heads[3]
                assert bool((y[b] == 0).all()) == behind, (over, b, more)


@pytest.mark.parametrize("io", ["f32", "bf16"])
@pytest.mark.parametrize("heads", HEADS, ids=lambda h: "x".join(map(str, h)))
def test_append_behind_the_last_page(ssd, heads, io):  # noqa: F811
    H, Hk, D, page = heads
    for single in (False, True):
        over, new = [3, None, 1, 70], [1, 1, 1, 1] if single else [5, 9, 1, 20]
        s, full = grown(heads, io, over, new, seed=7)
        g = torch.Generator().manual_seed(8)
        tokens = sum(new)
        q, k, v = (torch.randn((tokens, h, D), generator=g).to(TYPES[io]) for h in (H, Hk, Hk))
        rope = rope_table(s["table"].shape[1] * page, D)
        d, given = dev(s), torch.full((tokens, H, D), 5.0, dtype=TYPES[io], device="cuda")
        print("append", heads, io, new, flush=True)
        q_out = ssd.ssd_attn_append(q.cuda(), k.cuda(), v.cuda(), d["k"], d["v"], d["table"], d["lens"], None if single else d["cu"],
                                    rope=[t.cuda() for t in rope], q_out=given).cpu()
        torch.cuda.synchronize()
        kept = torch.zeros_like(s["k"], dtype=torch.bool)
        at = 0
        for b, n in enumerate(new):
            for j in range(n):
                pos = int(s["lens"][b]) - n + j
                if pos < full:
                    where = int(s["table"][b, pos // page]), slice(None), pos % page
                    kept[where] = True
                    assert torch.equal(d["v"].cpu()[where], v[at])
                else:
                    assert bool((q_out[at] == 5).all()), (b, j)
                at += 1
        for name in ("k", "v"):   # nobody else's slots are written
            same = (d[name].cpu() == s[name]) | (s[name].isnan() & d[name].cpu().isnan())
            assert bool((same | kept).all()), name


def test_a_captured_step_that_outgrows_its_row(ssd):  # noqa: F811
    """Append and step captured once, replayed past the end of a sequence's row: what it holds stays, and its y is 0."""
    H, Hk, D, page = 8, 2, 128, 16
    s = make([48, 48], H, Hk, D, page, "bf16", seed=3)
    s["table"][1] = s["table"][0]           # a page shared by two sequences, of which the other one is shorter
    d = dev(s)
    lens = torch.tensor([45, 20], dtype=torch.int32, device="cuda")
    q, k, v = (torch.randn((2, h, D), device="cuda").bfloat16() for h in (H, Hk, Hk))
    d["table"][1, 1:] = -1                  # (the second one appends nothing)
    q_out, y = torch.zeros_like(q), torch.empty_like(q)
    rope = [t.cuda() for t in rope_table(48, D)]
    ws = torch.empty(max(256, ssd.attn_step_workspace_bytes(ssd.make_attn_shape(2, 2, H, d["k"], d["table"]))), dtype=torch.uint8, device="cuda")

    def step():
        ssd.ssd_attn_append(q, k, v, d["k"], d["v"], d["table"], lens, rope=rope, q_out=q_out)
        ssd.ssd_attn_step(q_out, d["k"], d["v"], d["table"], lens, y=y, workspace=ws)

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=torch.cuda.Stream()):
        step()
    for length in range(46, 53):
        lens[0] = length
        before = d["k"].clone(), d["v"].clone()
        graph.replay()
        torch.cuda.synchronize()
        if length <= 48:
            assert bool((y[0] != 0).any()) and not torch.equal(d["v"].view(torch.int16), before[1].view(torch.int16)), length
        else:
            assert bool((y[0] == 0).all()), length
            assert torch.equal(d["k"].view(torch.int16), before[0].view(torch.int16)), length
            assert torch.equal(d["v"].view(torch.int16), before[1].view(torch.int16)), length
        assert bool((y[1] != 0).any())
