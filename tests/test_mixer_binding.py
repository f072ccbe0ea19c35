"""The native marshalling of the packed convolution, the selective scan and the append with normed heads: it answers None where
anything is out of the ordinary, and where it takes a call the results are those of the Python path, bit for bit."""
import types

import pytest
import torch

from paper_2603_09555_amd import ssd

ARGS = {"conv1d_varlen": 9, "selective_prefill": 15, "selective_step": 12, "attn_append_norm": 14}


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
    f, cu = torch.float32, i(0, 4, 4, 9)
    yield "ssd_conv1d_varlen", (n(9, 40)[:, 3:27], n(24, 4, dt=f), n(24, dt=f), cu), {}
    yield "ssd_conv1d_varlen", (n(9, 24), n(24, 3, dt=f), None, cu, n(3, 24, 2)), dict(split=(16, 0, 8), activation="none", outs=[n(9, 16), n(9, 8)],
                                                                                       conv_state_out=n(3, 24, 2))
    yield "ssd_conv1d_varlen", (n(1, 24), n(24, 3, dt=f), None, i(0, 1)), dict(split=[24])
    scan = (n(9, 24), n(9, 24), -n(24, 5, dt=f).abs(), n(9, 30)[:, 4:9], n(9, 5), n(24, dt=f))
    yield "ssd_selective_prefill", (*scan, cu), dict(dt_softplus=True)
    yield "ssd_selective_prefill", (*scan, cu), dict(z=n(9, 50)[:, 26:], h0=n(3, 24, 5, dt=f), y=n(9, 24), final_state=n(3, 24, 5, dt=f), dt_softplus=True,
                                                     dt_bias=n(24, dt=f), dt_limit=(0.01, 0.2), workspace=torch.empty(1 << 20, dtype=torch.uint8, device="cuda"))
    yield "ssd_selective_prefill", (scan[0], scan[1].float(), *scan[2:5], None, cu), dict(dt_softplus=True)
    yield "ssd_selective_step", (n(9, 24, 5, dt=f), *scan), dict(dt_softplus=True, z=n(9, 24))
    yield "ssd_selective_step", (n(9, 24, 5, dt=f), *scan[:5], None), dict(dt_softplus=True, y=n(9, 24), dt_bias=n(24, dt=f), dt_limit=(0.01, 0.2))
    table, lens = torch.tensor([[1, 0], [4, 2], [3, 5]], dtype=torch.int32, device="cuda"), i(20, 3, 32)
    kc, vc, w = n(6, 2, 16, 64), n(6, 2, 16, 64), (n(64, dt=f), n(64, dt=f))
    rope = (n(40, 16, dt=f), n(40, 16, dt=f))
    q, k, v = (t.unflatten(1, (-1, 64)) for t in n(9, 8 * 64).split((256, 128, 128), dim=1))
    yield "ssd_attn_append_norm", (q, k, v, *w, kc, vc, table, lens, cu), dict(rope=rope)
    yield "ssd_attn_append_norm", (q, k, v, *w, kc, vc, table, lens, cu), dict(rope=list(rope), interleaved=True, eps=0.5, q_out=n(9, 4, 64))
    yield "ssd_attn_append_norm", (None, n(3, 2, 64), n(3, 2, 64), None, w[1], kc, vc, table, lens), {}


def _flat(out):
    if out is None:
        return []
    return [t for o in out for t in _flat(o)] if isinstance(out, (tuple, list)) else [out]


def _cloned(v):
    if isinstance(v, list):
        return [_cloned(t) for t in v]
    return v.clone() if isinstance(v, torch.Tensor) and v.is_contiguous() else v   # (slices are read only)


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
            print(name, use, flush=True)
            out = getattr(ssd, name)(*a, **k)
            torch.cuda.synchronize()
            tensors = [t for t in a + list(k.values()) if isinstance(t, torch.Tensor) and t.dtype != torch.uint8]
            got.append([t.clone() for t in _flat(out) + tensors])
        assert taken[0] is not None and taken[1] is None, name
        assert len(got[0]) == len(got[1])
        for x, y in zip(*got):
            assert torch.equal(x, y), name
