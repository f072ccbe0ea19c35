"""The native marshalling of the norms and of the operators on a paged cache: it answers None where anything is out of the
ordinary, and where it takes a call the results are those of the Python path, bit for bit."""
import types

import pytest
import torch

from paper_2603_09555_amd import ssd

ARGS = {"norm_gated": 7, "norm_residual": 7, "attn_append": 11, "attn_step": 9, "attn_prefill": 10}


@pytest.mark.parametrize("name", sorted(ARGS))
def test_anything_but_device_tensors_is_left_to_python(name):
    f = getattr(ssd._native, name)
    t = torch.zeros(2, 2, 2, 2)
    assert f() is None
    for arg in (None, 3, "x", t, torch.nn.Parameter(t)):
        assert f(*[arg] * ARGS[name]) is None


def _calls(io):
    g = torch.Generator(device="cuda").manual_seed(9)
    n = lambda *s, dt=io: torch.randn(s, generator=g, device="cuda").to(dt)   # noqa: E731
    i = lambda *v: torch.tensor(v, dtype=torch.int32, device="cuda")          # noqa: E731
    f = torch.float32
    wide = n(5, 130)
    yield "ssd_norm_gated", (n(5, 64), wide[:, :64], n(64, dt=f)), {}
    yield "ssd_norm_gated", (n(5, 64), n(5, 64), n(64, dt=f)), dict(eps=1e-3, groups=2, norm_first=True, out=n(5, 64))
    yield "ssd_norm_gated", (n(1, 64), n(1, 64), n(64, dt=f)), {}
    yield "ssd_norm_residual", (n(5, 64, dt=f), n(5, 64), n(64, dt=f)), dict(scale=0.5)
    yield "ssd_norm_residual", (None, n(5, 64), n(64, dt=f)), {}
    yield "ssd_norm_residual", (n(5, 64), n(5, 64), n(64, dt=f)), dict(out=n(5, 64), residual_out=n(5, 64))
    yield "ssd_norm_residual", (None, n(5, 64), n(64, dt=f)), dict(residual_out=n(5, 64))
    table, lens, cu = torch.tensor([[1, 0], [4, 2], [3, 5]], dtype=torch.int32, device="cuda"), i(20, 3, 32), i(0, 4, 4, 9)
    kc, vc = n(6, 2, 16, 64), n(6, 2, 16, 64)
    rope = (n(40, 16, dt=f), n(40, 16, dt=f))
    qkv = n(9, 8 * 64)
    q, k, v = (t.unflatten(1, (-1, 64)) for t in qkv.split((256, 128, 128), dim=1))
    yield "ssd_attn_append", (q, k, v, kc, vc, table, lens, cu), dict(rope=rope)
    yield "ssd_attn_append", (q, k, v, kc, vc, table, lens, cu), dict(rope=list(rope), interleaved=True, q_out=n(9, 4, 64))
    yield "ssd_attn_append", (None, n(3, 2, 64), n(3, 2, 64), kc, vc, table, lens), {}
    yield "ssd_attn_append", (n(3, 4, 64), n(3, 2, 64), n(3, 2, 64), kc, vc, table, lens), {}
    yield "ssd_attn_step", (n(3, 4, 64), kc, vc, table, lens), {}
    yield "ssd_attn_step", (n(3, 4, 64), kc, vc, table, lens), dict(scale=0.25, window=7, y=n(3, 4, 64),
                                                                   workspace=torch.empty(1 << 24, dtype=torch.uint8, device="cuda"))
    yield "ssd_attn_prefill", (n(9, 4, 64), kc, vc, table, lens, cu), {}
    yield "ssd_attn_prefill", (n(9, 4, 64), kc, vc, table, lens, cu), dict(scale=0.25, window=7, y=n(9, 4, 64))


def _flat(out):
    return [] if out is None else list(out) if isinstance(out, tuple) else [out]


def _cloned(v):
    if isinstance(v, torch.Tensor):
        return v.clone() if v.is_contiguous() else v   # (slices are read only)
    return v


@pytest.mark.gpu
@pytest.mark.parametrize("io", [torch.bfloat16, torch.float32], ids=str)
def test_both_paths_agree(io, monkeypatch):
    native = ssd._native
    for name, args, kw in _calls(io):
        got, taken = [], []
        for use in (True, False):
            fs = {n: (lambda *a, n=n: taken.append(getattr(native, n)(*a) if use else None) or taken[-1]) for n in ARGS}
            monkeypatch.setattr(ssd, "_native", types.SimpleNamespace(**fs))
            a, k = [_cloned(v) for v in args], {n: _cloned(v) for n, v in kw.items()}
            out = getattr(ssd, name)(*a, **k)
            torch.cuda.synchronize()
            given = k.get("y", k.get("q_out", k.get("out")))
            assert given is None or _flat(out)[0] is given, name
            got.append(_flat(out) + [v for v in a if isinstance(v, torch.Tensor)])
        assert taken[0] is not None and taken[1] is None and len(taken) == 2, name
        assert len(got[0]) == len(got[1]) and all(s.dtype == t.dtype and torch.equal(s, t) for s, t in zip(*got)), name


@pytest.mark.gpu
def test_wrong_tensors_are_refused_by_both():
    """A tensor of another type, a size that doesn't fit, or not dense: neither path makes the call."""
    for name, args, kw in _calls(torch.bfloat16):
        for at, t in enumerate(args):
            if not isinstance(t, torch.Tensor):
                continue
            other = {torch.float32: torch.bfloat16, torch.bfloat16: torch.float32, torch.int32: torch.int64}[t.dtype]
            for what, v in (("type", t.to(other)), ("size", t[..., :-1].contiguous()), ("strides", torch.stack([t, t], -1)[..., 0])):
                # (calls of their own: a stream in another type, rows in fp32, a page table of fewer columns)
                if (name == "ssd_norm_residual" and at < 2 and what == "type") or (t.dtype == torch.int32 and t.dim() == 2 and what == "size"):
                    continue
                a = list(args)
                a[at] = v
                with pytest.raises((ValueError, ssd.SSDError)):
                    getattr(ssd, name)(*a, **kw)


@pytest.mark.gpu
def test_a_failing_call_raises_its_status():
    z = torch.zeros(3, 3, 64, device="cuda")
    cache, table, lens = torch.zeros(2, 2, 16, 64, device="cuda"), torch.zeros(3, 1, dtype=torch.int32, device="cuda"), torch.zeros(3, dtype=torch.int32, device="cuda")
    with pytest.raises(ssd.SSDError) as e:   # three heads over two key heads
        ssd.ssd_attn_step(z, cache, cache, table, lens)
    assert e.value.status == -2
    with pytest.raises(ssd.SSDError) as e:   # a rotation table that is too short
        ssd.ssd_attn_append(None, z[:, :2].contiguous(), z[:, :2].contiguous(), cache, cache, table, lens, rope=(torch.zeros(15, 8, device="cuda"),) * 2)
    assert e.value.status == -2
