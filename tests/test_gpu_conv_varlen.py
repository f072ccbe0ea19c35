"""The convolution of packed prompts: every bit that of the batched one on each sequence by itself, and within rounding of its
definition in fp64.

Limits: the sum of k products and a bias rounds k times, relative to the sum of its terms' absolute values; SiLU's slope is below
1.1, its exponential's argument is rounded twice (2 |a| u) and three more roundings follow, u = 2^-24; the result is rounded once."""
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


def make(lengths, split, k, io, seed, gaps=(0, 0), pad=0, cached=True, bias=True):
    g = torch.Generator().manual_seed(seed)
    C, t = sum(split), sum(lengths) + sum(gaps)
    wide = torch.randn((t, pad + C + pad), generator=g).to(IO[io])
    return dict(wide=wide, pad=pad, u=wide[:, pad:pad + C], w=torch.randn((C, k), generator=g) / k, b=0.1 * torch.randn((C,), generator=g) if bias else None,
                cu=torch.tensor([gaps[0]] + lengths).cumsum(0).to(torch.int32),
                state=torch.randn((len(lengths), C, k - 1), generator=g).to(IO[io]) if cached else None)


def call(ssd, s, split, act="silu", in_place=False):
    dev = lambda t: None if t is None else t.cuda()   # noqa: E731
    u = s["wide"].cuda()[:, s["pad"]:s["pad"] + sum(split)]
    outs = [torch.full((u.shape[0], w), 5.0, dtype=u.dtype, device="cuda") for w in split if w]
    state = dev(s["state"])
    got, new = ssd.ssd_conv1d_varlen(u, dev(s["w"]), dev(s["b"]), dev(s["cu"]), state, split=split, activation=act, outs=outs,
                                     conv_state_out=state if in_place else None)
    torch.cuda.synchronize()
    assert got is outs and (not in_place or new is state)
    return torch.cat(got, dim=1), new


def compare(ssd, s, split, k, io, act):
    z, new = call(ssd, s, split, act)
    ref, caches = mixer_oracle.conv1d_varlen(s["u"], s["w"], s["b"], s["cu"], s["state"], act, z=np.full(s["u"].shape, 5.0))
    a = mixer_oracle.conv1d_varlen(s["u"], s["w"], s["b"], s["cu"], s["state"], "none", z=np.zeros(s["u"].shape))[0]
    mag = mixer_oracle.conv1d_varlen(s["u"].abs(), s["w"].abs(), None if s["b"] is None else s["b"].abs(), s["cu"],
                                     None if s["state"] is None else s["state"].abs(), "none", z=np.zeros(s["u"].shape))[0]
    half = torch.finfo(IO[io]).eps / 2
    limit = half * np.abs(ref) * (1 + half) + 1.1 * (k + 1) * U * mag + (2 * np.abs(a) + 4) * U * np.abs(ref)
    got = z.double().cpu().numpy()
    worst = np.max(np.abs(got - ref) / np.maximum(limit, 1e-300), where=ref != 5.0, initial=0.0)
    print("conv %.3f of the limit" % worst, flush=True)
    assert worst <= 1.0
    assert np.array_equal(new.double().cpu().numpy(), caches), "the cache is a copy of inputs"
    lo, hi = int(s["cu"][0]), int(s["cu"][-1])
    assert (z[:lo] == 5).all() and (z[hi:] == 5).all()
    # every sequence by itself
    dev = lambda t: None if t is None else t.cuda()   # noqa: E731
    for q, (b, e) in enumerate(zip(s["cu"].tolist(), s["cu"].tolist()[1:])):
        if e > b:
            one, _ = ssd.ssd_conv1d_prefill(s["u"][None, b:e].contiguous().cuda(), s["w"].cuda(), dev(s["b"]),
                                            None if s["state"] is None else s["state"][q:q + 1].cuda().clone(), split=split, activation=act)
            assert torch.equal(torch.cat(one, dim=2)[0], z[b:e]), q
    return z, new


@pytest.mark.parametrize("io", ["f32", "bf16"])
@pytest.mark.parametrize("split,k", [((64,), 4), ((128, 32, 32), 4), ((24, 8, 8), 2), ((37,), 4), ((20, 3, 3), 3), ((6, 0, 5), 8), ((1,), 4), ((512, 128, 128), 5)])
def test_packed_prompts(ssd, split, k, io):
    for i, lengths in enumerate(([1], [2, 0, 9], [0], [0, 1, 1, 300, 0, 47, 0], [3] * 90)):
        s = make(lengths, split, k, io, seed=i, gaps=((0, 0), (3, 0), (0, 2), (1, 4), (0, 0))[i], pad=(0, 1, 8, 3, 0)[i], cached=i != 3, bias=i != 4)
        print("conv", split, k, io, lengths[:8], flush=True)
        z, new = compare(ssd, s, split, k, io, "none" if i == 1 else "silu")
        if s["state"] is not None:
            z2, new2 = call(ssd, s, split, "none" if i == 1 else "silu", in_place=True)
            assert torch.equal(z2, z) and torch.equal(new2, new)


def test_long_prompts(ssd):
    compare(ssd, make([2000, 1, 777, 0, 3001], (384, 64, 64), 4, "bf16", seed=9, pad=4), (384, 64, 64), 4, "bf16", "silu")


def test_boundaries_that_no_batch_has(ssd):
    s = make([100, 200], (64,), 4, "f32", seed=10)
    for cu in ([-7, 100, 400], [-5, -3, 300], [300, 300, 301], [0, 0, 2 ** 31 - 1], [-2 ** 31, 50, 50]):
        t = dict(s, cu=torch.tensor(cu, dtype=torch.int32))
        print("boundaries", cu, flush=True)
        z, new = call(ssd, t, (64,))
        ref, caches = mixer_oracle.conv1d_varlen(t["u"], t["w"], t["b"], t["cu"], t["state"], z=np.full(t["u"].shape, 5.0))
        assert np.allclose(z.double().cpu().numpy(), ref, rtol=1e-5, atol=1e-5) and np.array_equal(new.double().cpu().numpy(), caches)
    for cu in ([200, 100, 0], [0, 300, 100], [250, 20, 280]):
        call(ssd, dict(s, cu=torch.tensor(cu, dtype=torch.int32)), (64,))


def test_captured(ssd):
    s, t = make([100, 3, 200], (64, 8), 4, "bf16", seed=11), make([1, 280, 22], (64, 8), 4, "bf16", seed=12)
    u, w, b, cu, state = (v.cuda().clone() for v in (s["u"], s["w"], s["b"], s["cu"], s["state"]))
    outs = [torch.empty((303, n), dtype=torch.bfloat16, device="cuda") for n in (64, 8)]
    graph = torch.cuda.CUDAGraph()
    call_it = lambda: ssd.ssd_conv1d_varlen(u, w, b, cu, state, split=(64, 8), outs=outs, conv_state_out=state)   # noqa: E731
    call_it()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        call_it()
    for v in (s, t, t, s):
        for to, name in ((u, "u"), (w, "w"), (b, "b"), (cu, "cu"), (state, "state")):
            to.copy_(v[name])
        graph.replay()
        torch.cuda.synchronize()
        z, new = call(ssd, v, (64, 8), in_place=True)
        assert torch.equal(torch.cat(outs, dim=1), z) and torch.equal(state, new)


def test_more_sequences_than_fit_lds(ssd):
    compare(ssd, make([1, 2, 0, 5] * 400, (20, 4), 4, "bf16", seed=13, gaps=(2, 1)), (20, 4), 4, "bf16", "silu")
    compare(ssd, make([3, 0] * 600, (5,), 3, "f32", seed=14, gaps=(0, 7)), (5,), 3, "f32", "none")


def test_offsets_beyond_32_bits(ssd):
    """4.4 GiB of input: rows around 2 and 4 GiB and at the end are those of the batched call on slices."""
    T, C = 288000, 8192
    g = torch.Generator(device="cuda").manual_seed(15)
    u = torch.randn((T, C), generator=g, device="cuda", dtype=torch.bfloat16)
    w, b = torch.randn((C, 4), generator=g, device="cuda") / 4, torch.randn((C,), generator=g, device="cuda")
    cu = torch.tensor([0, 1000, 262200, T], dtype=torch.int32, device="cuda")
    print("conv", T, C, flush=True)
    (z,), new = ssd.ssd_conv1d_varlen(u, w, b, cu)
    torch.cuda.synchronize()
    for at in (131072, 262144, T):
        lo = at - 64
        one, state = ssd.ssd_conv1d_prefill(u[None, lo - 3:at].contiguous(), w, b)
        assert torch.equal(z[lo:at], one[0][0, 3:]), at
    assert torch.equal(new[2], u[T - 3:].t())
    assert torch.equal(z[262200:262203], ssd.ssd_conv1d_prefill(u[None, 262200:262203].contiguous(), w, b)[0][0][0])
