"""The selective scan against its fp64 oracle, element by element.

Limits are those of a rounding analysis, relative to the sum of the absolute values of a result's terms (``magnitude`` of the
oracle), with u = 2^-24 a rounding of fp32.  A token multiplies a state by exp(d A), which carries 2 u of the hardware's exponential
and, |d A| e^-|d A| <= 0.37 being what an error of the exponent counts for, some 3 u from the exponent (A log2(e) and its product
rounded, the step size within 4 u); the sum behind it rounds once more.  6 u a token, over the L tokens that a state has seen
(the sum of a stretch's step sizes, L roundings at most, is within that); 32 u for the inflow, the skip term and the gate's
reciprocal, N u for the sum over states, 2 |z| u for the gate's exponential (its argument is rounded twice).  The result is rounded once, by
half of eps."""
import numpy as np
import pytest
import torch

from oracle import mixer_oracle, ssd_oracle

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
IO = {"f32": torch.float32, "bf16": torch.bfloat16}


@pytest.fixture(scope="module")
def ssd():
    from paper_2603_09555_amd import ssd as binding
    return binding


def make(lengths, C, N, io, dt="same", seed=0, gate=True, skip=True, cached=True, gaps=(0, 0), pad=(5, 3), steps=1.0):
    """Inputs on the host; B, C and z are slices of wider rows.  ``gaps``: tokens in front of the first and behind the last sequence."""
    g = torch.Generator().manual_seed(seed)
    t = sum(lengths) + sum(gaps)
    iod = IO[io]
    n = lambda *s, scale=1.0, dt=iod: (scale * torch.randn(s, generator=g)).to(dt)   # noqa: E731
    cu = torch.tensor([gaps[0]] + lengths, dtype=torch.int64).cumsum(0).to(torch.int32)
    bc, xz = n(t, pad[0] + 2 * N + pad[1], scale=0.5), n(t, C + pad[1])
    f32 = torch.float32
    return dict(x=n(t, C), dt=n(t, C, scale=0.5, dt=f32 if dt == "f32" else iod), A=-torch.rand((C, N), generator=g) * 15.5 - 0.5,
                B=bc[:, pad[0]:pad[0] + N], C=bc[:, pad[0] + N:pad[0] + 2 * N], D=n(C, dt=f32) if skip else None, z=xz[:, pad[1]:] if gate else None,
                cu=cu, h0=n(len(lengths), C, N, dt=f32) if cached else None,
                dt_bias=torch.log(torch.expm1(torch.rand((C,), generator=g) * 0.1 * steps + 1e-3)))


def to_gpu(t):
    if t is None or t.is_contiguous():
        return None if t is None else t.cuda()
    base = t._base.cuda()
    return base.as_strided(t.shape, t.stride(), t.storage_offset())


def limits(s, d, y_ref, h_ref, io, length):
    """Allowed errors of y and of the final states."""
    ym, hm = mixer_oracle.selective_scan(s["x"], d, s["A"], s["B"], s["C"], s["D"], s["cu"], s["z"], s["h0"], magnitude=True)
    z = 0.0 if s["z"] is None else np.abs(s["z"].double().numpy())
    half = torch.finfo(IO[io]).eps / 2
    return half * np.abs(y_ref) * (1 + half) + (6 * length + s["A"].shape[1] + 32 + 2 * z) * U * ym, (6 * length + 32) * U * hm


def check(got, ref, limit, what):
    got = got.detach().double().cpu().numpy()
    there = ~np.isnan(ref)
    assert np.isfinite(got[there]).all(), what
    worst = np.max(np.abs(got - ref)[there] / np.maximum(limit[there], 1e-300), initial=0.0)
    print("%s: %.3f of the limit" % (what, worst), flush=True)
    assert worst <= 1.0, what


def run(ssd, s, limit=None, **kw):
    d = {k: to_gpu(v) for k, v in s.items()}
    y = torch.full_like(d["x"], 7.0)
    y, f = ssd.ssd_selective_prefill(d["x"], d["dt"], d["A"], d["B"], d["C"], d["D"], d["cu"], z=d["z"], h0=d["h0"], y=y, dt_bias=d["dt_bias"],
                                     dt_softplus=True, dt_limit=limit, **kw)
    torch.cuda.synchronize()
    return y, f


def compare(ssd, s, io, limit=None):
    d = ssd_oracle.dt_transform(s["dt"], s["dt_bias"], True, limit)
    y_ref, h_ref = mixer_oracle.selective_scan(s["x"], d, s["A"], s["B"], s["C"], s["D"], s["cu"], s["z"], s["h0"],
                                               y=np.full(s["x"].shape, 7.0))
    ly, lh = limits(s, d, y_ref, h_ref, io, int(np.diff(s["cu"].numpy()).max()))
    lo, hi = int(s["cu"][0]), int(s["cu"][-1])
    y, f = run(ssd, s, limit)
    check(y[lo:hi], y_ref[lo:hi], ly[lo:hi], "y")
    check(f, h_ref, lh, "states")
    assert (y[:lo] == 7).all() and (y[hi:] == 7).all(), "tokens of no sequence are left as they were"
    return y, f


@pytest.mark.parametrize("io,dt", [("f32", "same"), ("bf16", "same"), ("bf16", "f32")])
@pytest.mark.parametrize("C,N", [(64, 16), (1, 1), (65, 7), (130, 8), (63, 13), (200, 16), (7, 24), (96, 32), (40, 33), (64, 64), (3, 100), (70, 128), (66, 256)])
def test_prompts(ssd, C, N, io, dt):
    for i, lengths in enumerate(([1], [2, 0, 9], [0], [63, 64, 65], [0, 300, 0, 0, 31, 0])):
        print("selective", C, N, io, dt, lengths, flush=True)
        s = make(lengths, C, N, io, dt, seed=i, gate=i % 2 == 0, skip=i != 2, cached=i != 3, gaps=((0, 0), (3, 0), (0, 2), (1, 4), (0, 0))[i],
                 pad=(i, 4 * i))
        compare(ssd, s, io, limit=(1e-3, 0.1) if i == 1 else None)


@pytest.mark.parametrize("io", ["f32", "bf16"])
@pytest.mark.parametrize("aligned", [True, False])
def test_long_prompts_of_few_channels(ssd, io, aligned):
    """Many segments, that begin and end anywhere in sequences."""
    for i, lengths in enumerate(([1500], [700, 1, 0, 900, 2], [3] * 200 + [800])):
        print("selective", io, aligned, lengths[:5], flush=True)
        s = make(lengths, 70, 16, io, seed=20 + i, pad=(2, 2) if aligned else (1, 2))
        compare(ssd, s, io)
        for segment in (200, 10000):
            ssd.set_knob("selective_segment", segment)
            compare(ssd, s, io)
        ssd.reset_knobs()


@pytest.mark.parametrize("C,N", [(4000, 16), (1000, 16), (900, 6), (700, 30), (400, 60), (130, 256)])
def test_every_cut(ssd, C, N):
    """More or fewer states a wave, by how much work there is."""
    for tokens in (81, 330):
        print("selective", C, N, tokens, flush=True)
        compare(ssd, make([tokens - 20, 0, 20], C, N, "bf16", seed=C + N), "bf16")


def test_decays_of_every_size(ssd):
    """Steps from nothing to ones that leave nothing of a state."""
    s = make([400], 64, 16, "f32", seed=30)
    s["dt"] = torch.randn((400, 64), generator=torch.Generator().manual_seed(31)) * 12.0
    s["A"][:, 0], s["A"][:, 1] = 0.0, -1e6
    compare(ssd, s, "f32")


def test_final_states_in_place(ssd):
    """Sequences that begin in one segment and end in another, states updated where they are."""
    s = make([5, 900, 0, 300, 299, 1], 64, 16, "bf16", seed=40)
    y, f = run(ssd, s)
    s2 = dict(s)
    held = s["h0"].cuda()
    d = {k: to_gpu(v) for k, v in s2.items()}
    for _ in range(2):
        held.copy_(s["h0"])
        y2, f2 = ssd.ssd_selective_prefill(d["x"], d["dt"], d["A"], d["B"], d["C"], d["D"], d["cu"], z=d["z"], h0=held, final_state=held,
                                           dt_bias=d["dt_bias"], dt_softplus=True)
        torch.cuda.synchronize()
        assert f2 is held and torch.equal(f2, f) and torch.equal(y2, y)


def test_boundaries_that_no_batch_has(ssd):
    """Boundaries outside the tokens are cut to them; what decreases gives anything, within the tensors."""
    s = make([100, 200], 64, 16, "f32", seed=50)
    for cu in ([-7, 100, 400], [-5, -3, 300], [300, 300, 301], [0, 0, 2 ** 31 - 1], [-2 ** 31, 50, 50]):
        t = dict(s, cu=torch.tensor(cu, dtype=torch.int32))
        print("boundaries", cu, flush=True)
        d = ssd_oracle.dt_transform(t["dt"], t["dt_bias"], True)
        args = (t["x"], d, t["A"], t["B"], t["C"], t["D"], t["cu"], t["z"], t["h0"])
        y_ref, h_ref = mixer_oracle.selective_scan(*args, y=np.full(t["x"].shape, 7.0))
        ly, lh = limits(t, d, y_ref, h_ref, "f32", 300)
        y, f = run(ssd, t)
        check(y, y_ref, np.where(np.isnan(ly), 0.0, ly), "y")
        check(f, h_ref, lh, "states")
    for cu in ([200, 100, 0], [0, 300, 100], [250, 20, 280]):
        print("boundaries", cu, flush=True)
        y, f = run(ssd, dict(s, cu=torch.tensor(cu, dtype=torch.int32)))
        assert y.shape == s["x"].shape


def test_what_a_sequence_does_not_hold_is_not_used(ssd):
    """Rows of no sequence, and other sequences, may hold anything."""
    s = make([70, 130], 65, 16, "f32", seed=60, gaps=(9, 11))
    y, f = run(ssd, s)
    bad = {k: s[k].clone() for k in ("x", "dt", "B", "C", "z")}
    for t in bad.values():
        t[:9] = float("nan")
        t[79:] = float("inf")
    s2 = dict(s, **bad)
    s2["h0"] = s["h0"].clone()
    s2["h0"][1] = float("nan")
    y2, f2 = run(ssd, s2)
    assert torch.equal(y2[9:79], y[9:79]) and torch.equal(f2[0], f[0])


@pytest.mark.parametrize("io,dt", [("f32", "same"), ("bf16", "same"), ("bf16", "f32")])
@pytest.mark.parametrize("C,N", [(64, 16), (1, 1), (65, 7), (130, 8), (200, 16), (7, 24), (96, 32), (3, 100), (70, 128), (5, 256)])
def test_steps(ssd, C, N, io, dt):
    for batch in (1, 3, 67):
        s = make([1] * batch, C, N, io, dt, seed=batch, gate=batch != 3, skip=batch != 67)
        print("step", C, N, io, dt, batch, flush=True)
        d = ssd_oracle.dt_transform(s["dt"], s["dt_bias"], True, (1e-3, 0.08))
        y_ref, h_ref = mixer_oracle.selective_scan(s["x"], d, s["A"], s["B"], s["C"], s["D"], s["cu"], s["z"], s["h0"])
        ly, lh = limits(s, d, y_ref, h_ref, io, 1)
        g = {k: to_gpu(v) for k, v in s.items()}
        y = ssd.ssd_selective_step(g["h0"], g["x"], g["dt"], g["A"], g["B"], g["C"], g["D"], z=g["z"], dt_bias=g["dt_bias"], dt_softplus=True,
                                   dt_limit=(1e-3, 0.08))
        torch.cuda.synchronize()
        check(y, y_ref, ly, "y")
        check(g["h0"], h_ref, lh, "states")


def test_plain_steps(ssd):
    """Step sizes used as they are given, zero among them (a state stays as it is)."""
    s = make([40], 64, 16, "f32", seed=70)
    s["dt"] = s["dt"].abs()
    s["dt"][10:20] = 0.0
    g = {k: to_gpu(v) for k, v in s.items()}
    y, f = ssd.ssd_selective_prefill(g["x"], g["dt"], g["A"], g["B"], g["C"], g["D"], g["cu"], z=g["z"], h0=g["h0"])
    state = g["h0"].clone()
    for t in range(40):
        kept = state.clone()
        yt = ssd.ssd_selective_step(state, *(g[k][t:t + 1].contiguous() for k in ("x", "dt")), g["A"], g["B"][t:t + 1], g["C"][t:t + 1], g["D"],
                                    z=g["z"][t:t + 1])
        assert not 10 <= t < 20 or torch.equal(state, kept)
    y_ref, h_ref = mixer_oracle.selective_scan(s["x"], s["dt"].double().numpy(), s["A"], s["B"], s["C"], s["D"], s["cu"], s["z"], s["h0"])
    ly, lh = limits(s, s["dt"].double().numpy(), y_ref, h_ref, "f32", 40)
    check(y, y_ref, ly, "y")
    check(f, h_ref, lh, "states")
    check(state[0], h_ref[0], lh[0], "states, step by step")
    check(yt[0], y_ref[39], ly[39], "y of the last step")


def test_captured_and_on_other_streams(ssd):
    """A captured call follows the boundaries as the device has them, and two graphs do not share what they leave."""
    a, b = make([600, 40, 160], 70, 16, "bf16", seed=80), make([10, 700, 90], 70, 16, "bf16", seed=81)
    ga, gb = ({k: to_gpu(v) for k, v in s.items()} for s in (a, b))
    want = [run(ssd, s) for s in (a, b)]
    held = {k: to_gpu(v) for k, v in a.items()}
    y, f = torch.empty_like(held["x"]), torch.empty_like(held["h0"])
    work = torch.empty(max(256, ssd.selective_prefill_workspace_bytes(ssd.make_selective_shape(3, 800, 70, 16, torch.bfloat16))), dtype=torch.uint8,
                       device="cuda")

    def call():
        ssd.ssd_selective_prefill(held["x"], held["dt"], held["A"], held["B"], held["C"], held["D"], held["cu"], z=held["z"], h0=held["h0"], y=y,
                                  final_state=f, workspace=work, dt_bias=held["dt_bias"], dt_softplus=True)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        call()
    torch.cuda.synchronize()
    assert torch.equal(y, want[0][0]) and torch.equal(f, want[0][1])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for turn in (0, 1, 0, 1, 1):
        s = (ga, gb)[turn]
        for k in ("x", "dt", "A", "D", "dt_bias", "cu", "h0"):
            held[k].copy_(s[k])
        for k in ("B", "C", "z"):
            held[k].copy_(s[k])
        y.fill_(3.0)
        work.fill_(255)
        graph.replay()
        torch.cuda.synchronize()
        ref = run(ssd, (a, b)[turn])
        assert torch.equal(y, ref[0]) and torch.equal(f, ref[1]), turn


@pytest.mark.parametrize("io", ["f32", "bf16"])
@pytest.mark.parametrize("N", [1, 7, 16, 24, 33, 64])
def test_both_kernels(ssd, N, io):
    """A lane a channel, and a lane a state, whatever the library would choose."""
    for i, lengths in enumerate(([300, 0, 1, 90], [17, 700])):
        s = make(lengths, 130, N, io, seed=90 + i, gaps=(i, 3 * i), pad=(1, 2))
        for kernel in (1, 2):
            ssd.set_knob("selective_by_state", kernel)
            print("selective", N, io, lengths, kernel, flush=True)
            y, f = compare(ssd, s, io)
            again = run(ssd, s)
            assert torch.equal(again[0][i:-3 * i or None], y[i:-3 * i or None]) and torch.equal(again[1], f)
        ssd.reset_knobs()


def test_many_sequences(ssd):
    """More sequences than channels, many of one token or none."""
    compare(ssd, make([1, 0, 2, 3, 1] * 300, 40, 16, "f32", seed=100, gaps=(1, 2)), "f32")


@pytest.mark.parametrize("kernel", [1, 2])
def test_offsets_beyond_32_bits(ssd, kernel):
    """4.4 GiB each of x, dt and y.  States forget within 60 tokens (exp(-60 x 0.5 x 4) is nothing in fp32), so that the oracle may start
    from zeros 120 tokens in front of what is compared."""
    T, C, N = 288000, 8192, 16
    g = torch.Generator(device="cuda").manual_seed(110)
    x = torch.randn((T, C), generator=g, device="cuda", dtype=torch.bfloat16)
    dt = torch.rand((T, C), generator=g, device="cuda", dtype=torch.bfloat16) + 0.5
    bc = torch.randn((T, 2 * N), generator=g, device="cuda", dtype=torch.bfloat16)
    A, D = -4.0 - torch.rand((C, N), generator=g, device="cuda"), torch.randn((C,), generator=g, device="cuda")
    cu = torch.tensor([0, 1000, T], dtype=torch.int32, device="cuda")
    ssd.set_knob("selective_by_state", kernel)
    print("selective", T, C, N, kernel, flush=True)
    y, f = ssd.ssd_selective_prefill(x, dt, A, bc[:, :N], bc[:, N:], D, cu)
    torch.cuda.synchronize()
    ssd.reset_knobs()
    for at in (131072 + 8, 262144 + 8, T):
        rows, cols = slice(at - 140, at), slice(C - 70, C)
        s = dict(x=x[rows, cols].cpu(), A=A[cols].cpu(), B=bc[rows, :N].cpu(), C=bc[rows, N:].cpu(), D=D[cols].cpu(), z=None, h0=None,
                 cu=torch.tensor([0, 140], dtype=torch.int32))
        d = dt[rows, cols].double().cpu().numpy()
        ref, h_ref = mixer_oracle.selective_scan(s["x"], d, s["A"], s["B"], s["C"], s["D"], s["cu"])
        ly, lh = limits(s, d, ref, h_ref, "bf16", 140)
        check(y[at - 20:at, cols], ref[-20:], ly[-20:], "y")
    check(f[1, cols], h_ref[0], lh[0], "states")


@pytest.mark.parametrize("by", [1, 2], ids=["by state", "by channel"])
@pytest.mark.parametrize("N", [5, 16, 40])
def test_states_that_keep_nothing(ssd, N, by):
    """A of -inf: exp(d A) is 0, and such a state is its last inflow, d x B; sequences end anywhere in a block of tokens, and segments
    in sequences.  The oracle multiplies 0 by what was there, so that its A of -1e30 says the same."""
    lengths = [1, 7, 0, 16, 90, 35]
    s = make(lengths, 70, N, "f32", seed=7)
    s["A"][::2, ::3] = float("-inf")
    ref = dict(s, A=torch.where(torch.isinf(s["A"]), torch.tensor(-1e30), s["A"]))
    d = ssd_oracle.dt_transform(s["dt"], s["dt_bias"], True, None)
    y_ref, h_ref = mixer_oracle.selective_scan(s["x"], d, ref["A"], s["B"], s["C"], s["D"], s["cu"], s["z"], s["h0"], y=np.full(s["x"].shape, 7.0))
    ly, lh = limits(ref, d, y_ref, h_ref, "f32", max(lengths))
    try:
        for segment in (0, 32):
            ssd.set_knob("selective_by_state", by)
            ssd.set_knob("selective_segment", segment)
            y, f = run(ssd, s)
            check(y, y_ref, ly, "y")
            check(f, h_ref, lh, "states")
    finally:
        ssd.reset_knobs()
    # single tokens of as many sequences
    batch = len(lengths)
    t1 = dict(ref, cu=torch.arange(batch + 1, dtype=torch.int32), **{k: s[k][:batch] for k in ("x", "dt", "B", "C", "z")})
    d = ssd_oracle.dt_transform(t1["dt"], s["dt_bias"], True, None)
    y_ref, h_ref = mixer_oracle.selective_scan(t1["x"], d, ref["A"], t1["B"], t1["C"], s["D"], t1["cu"], t1["z"], s["h0"])
    ly, lh = limits(t1, d, y_ref, h_ref, "f32", 1)
    state, g = s["h0"].cuda(), {k: to_gpu(s[k])[:batch] for k in ("x", "dt", "B", "C", "z")}
    y = ssd.ssd_selective_step(state, g["x"], g["dt"], s["A"].cuda(), g["B"], g["C"], s["D"].cuda(), z=g["z"], dt_bias=s["dt_bias"].cuda(),
                               dt_softplus=True)
    check(y, y_ref, ly, "y of a token")
    check(state, h_ref, lh, "states of a token")
