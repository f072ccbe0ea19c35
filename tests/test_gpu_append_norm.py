"""The append with normed heads against its fp64 oracle, element by element.

Limits: the sum of squares is made of runs of at most 8 values and 6 joins, the root halves its error, and mean, root, division,
scale, weight, rotation round some ten times more: 24 u with u = 2^-24, relative to the sum of the absolute values of the two
products of a rotation; rounded once, by half of eps."""
import numpy as np
import pytest
import torch

from oracle import mixer_oracle

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
IO = {"f32": torch.float32, "bf16": torch.bfloat16}


@pytest.fixture(scope="module")
def ssd():
    from paper_2603_09555_amd import ssd as binding
    return binding


def make(new, prior, H, Hk, D, page, rotary, io, seed, gaps=(0, 0), scale=1.0):
    g = torch.Generator().manual_seed(seed)
    lengths = [a + b for a, b in zip(new, prior)]
    width = max(1, max(-(-n // page) for n in lengths)) + 1
    t = sum(new) + sum(gaps)
    n = lambda *s, dt=IO[io]: torch.randn(s, generator=g).to(dt)   # noqa: E731
    npages = len(new) * width
    qkv = scale * n(t, (H + 2 * Hk) * D)
    angle = torch.rand((width * page, rotary // 2), generator=g) * 6
    return dict(qkv=qkv, heads=(H, Hk, Hk), D=D, qw=1 + 0.2 * torch.randn((D,), generator=g), kw=1 + 0.2 * torch.randn((D,), generator=g),
                kc=n(npages, Hk, page, D), vc=n(npages, Hk, page, D), table=torch.randperm(npages, generator=g).to(torch.int32).view(len(new), width),
                lens=torch.tensor(lengths, dtype=torch.int32), cu=torch.tensor([gaps[0]] + new).cumsum(0).to(torch.int32),
                rope=(angle.cos(), angle.sin()) if rotary else None, q_out=n(t, H, D))


def parts(s, qkv):
    return [t.unflatten(1, (-1, s["D"])) for t in qkv.split([h * s["D"] for h in s["heads"]], dim=1)]


def call(ssd, s, interleaved=False, cu=True, queries=True, eps=1e-5):
    q, k, v = parts(s, s["qkv"].cuda())
    kc, vc, out = s["kc"].cuda(), s["vc"].cuda(), s["q_out"].cuda()
    got = ssd.ssd_attn_append_norm(q if queries else None, k, v, s["qw"].cuda() if queries else None, s["kw"].cuda(), kc, vc, s["table"].cuda(),
                                   s["lens"].cuda(), s["cu"].cuda() if cu else None, rope=None if s["rope"] is None else tuple(t.cuda() for t in s["rope"]),
                                   interleaved=interleaved, eps=eps, q_out=out if queries else None)
    torch.cuda.synchronize()
    assert (got is out) if queries else got is None
    return got, kc, vc


def compare(ssd, s, io, interleaved=False, cu=True, queries=True, eps=1e-5):
    q, k, v = parts(s, s["qkv"])
    args = (q if queries else None, k, v, s["qw"], s["kw"], s["kc"], s["vc"], s["table"], s["lens"], s["cu"] if cu else None, s["rope"], interleaved, eps,
            s["q_out"] if queries else None)
    ref, mag = mixer_oracle.append_norm(*args), mixer_oracle.append_norm(*args, magnitude=True)
    got = call(ssd, s, interleaved, cu, queries, eps)
    half = torch.finfo(IO[io]).eps / 2
    for name, g, r, m, old in zip(("q", "k"), got, ref, mag, (s["q_out"], s["kc"])):
        if g is None:
            continue
        g, old = g.double().cpu().numpy(), old.double().numpy()
        written = r != old
        assert np.array_equal(g[~written], old[~written]), name
        worst = np.max(np.abs(g - r)[written] / (half * np.abs(r) * (1 + half) + 24 * U * np.abs(m))[written], initial=0.0)
        print("%s %.3f of the limit" % (name, worst), flush=True)
        assert worst <= 1.0, name
    assert np.array_equal(got[2].double().cpu().numpy(), ref[2]), "values are copied"


@pytest.mark.parametrize("io", ["f32", "bf16"])
@pytest.mark.parametrize("H,Hk,D,page,rotary", [(32, 8, 128, 16, 128), (4, 2, 64, 16, 32), (1, 1, 8, 1, 8), (5, 1, 80, 64, 40), (6, 3, 24, 8, 12), (2, 2, 256, 16, 256),
                                                (3, 1, 200, 4, 0), (16, 1, 96, 16, 66), (33, 11, 112, 32, 112)])
def test_packed_and_single_tokens(ssd, H, Hk, D, page, rotary, io):
    for i, (new, prior, gaps) in enumerate((([1], [0], (0, 0)), ([3, 0, 40, 1], [5, 9, 0, 70], (2, 3)), ([1, 1, 1], [4, 0, 33], (0, 0)))):
        for interleaved in (False, True):
            s = make(new, prior, H, Hk, D, page, rotary, io, seed=i, gaps=gaps)
            print("append", H, Hk, D, page, rotary, io, new, interleaved, flush=True)
            compare(ssd, s, io, interleaved, cu=i != 2, queries=not (i == 1 and interleaved), eps=1e-5 if i else 1e-2)


@pytest.mark.parametrize("io", ["f32", "bf16"])
def test_many_tokens(ssd, io):
    """Enough for several tokens a workgroup."""
    compare(ssd, make([1500, 0, 700], [3, 1, 30], 12, 4, 64, 16, 64, io, seed=5), io)


@pytest.mark.parametrize("scale", [1e-18, 1e15])
def test_small_and_large_heads(ssd, scale):
    compare(ssd, make([20], [2], 4, 2, 64, 16, 64, "f32", seed=6, scale=scale), "f32", eps=0.0 if scale > 1 else 1e-30)


def test_tokens_without_a_place(ssd):
    """In no sequence, in front of one, on pages that are not there: left out, and nothing else moves."""
    s = make([6, 9], [0, 4], 4, 2, 64, 4, 64, "f32", seed=7, gaps=(2, 2))
    s["lens"][0] = 4                         # two of its tokens are in front of its beginning
    s["table"][1, 1] = -1
    s["table"][1, 2] = s["kc"].shape[0]
    compare(ssd, s, "f32")
    s["lens"][1] = s["table"].shape[1] * 4 + 3   # three are behind its row of the table
    compare(ssd, s, "f32")


def test_without_norm_it_is_the_plain_append(ssd):
    """Heads that are normalised already (their squares' mean is exactly one) and weights of one."""
    s = make([33, 2], [1, 5], 4, 2, 64, 16, 64, "bf16", seed=8)
    s["qkv"] = torch.where(s["qkv"] > 0, 1.0, -1.0).to(torch.bfloat16)
    s["qw"], s["kw"] = torch.ones(64), torch.ones(64)
    got = call(ssd, s, eps=0.0)
    q, k, v = parts(s, s["qkv"].cuda())
    kc, vc = s["kc"].cuda(), s["vc"].cuda()
    out = ssd.ssd_attn_append(q, k, v, kc, vc, s["table"].cuda(), s["lens"].cuda(), s["cu"].cuda(), rope=tuple(t.cuda() for t in s["rope"]))
    for a, b in zip(got, (out, kc, vc)):
        assert torch.equal(a, b)
