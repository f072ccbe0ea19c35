"""What the packed convolution, the selective scan and the append with normed heads refuse, before any HIP call (so these run on
a CPU machine): through the C ABI, and through the Python binding on tensors that are never looked into."""
import ctypes

import pytest
import torch

from paper_2603_09555_amd import ssd

FAKE, HALF, ODD, FOUR = (ctypes.c_void_p(v) for v in (4096, 4098, 4097, 4100))   # never dereferenced: validation fails first


def refusals(call, null, align, elements):
    for name in null:
        assert call(**{name: None}) == -1, name
    for name in align:
        assert call(**{name: FOUR}) == -7, name
    for name in elements:
        assert call(**{name: ODD}) == -7, name


def test_conv_varlen_refuses():
    lib = ssd.raw()

    def call(batch=3, tokens=20, k=4, io=1, split=(32, 8, 8), cu=FAKE, u=FAKE, us=48, w=FAKE, bias=FAKE, si=FAKE, z0=FAKE, z1=FAKE, z2=FAKE, so=FAKE,
             act=1):
        return lib.ssd_conv1d_varlen(batch, tokens, k, io, None if split is None else (ctypes.c_int32 * 3)(*split), cu, u, us, w, bias, si, z0, z1, z2,
                                     so, act, None)

    for bad in (dict(batch=0), dict(tokens=0), dict(tokens=(1 << 30) + 1), dict(batch=(1 << 30) + 1), dict(k=1), dict(k=9), dict(split=(0, 8, 8)),
                dict(split=(8, -1, 8)), dict(us=47), dict(act=2), dict(us=1 << 60), dict(tokens=1 << 30, split=(1 << 20, 0, 0), us=1 << 20),
                dict(batch=1 << 26)):
        assert call(**bad) == -2, bad
    assert call(io=2) == -3
    refusals(call, ("split", "cu", "u", "w", "z0", "z1", "z2"), ("w", "bias", "si", "so", "z0", "z1", "z2"), ("u", "cu"))
    assert call(cu=HALF) == -7 and call(io=0, u=HALF) == -7


OK = dict(batch=3, tokens=20, channels=96, dstate=16, io_dtype=1, dt_dtype=1)
BAD = [(dict(batch=0), -2), (dict(channels=0), -2), (dict(dstate=0), -2), (dict(dstate=257), -4), (dict(io_dtype=2), -3), (dict(io_dtype=0), -3),
       (dict(dt_dtype=2), -3), (dict(channels=(1 << 22) + 1), -2), (dict(batch=2 ** 31 - 1), -2)]


def shape(**kw):
    return ssd.ssd_selective_shape(**dict(OK, **kw))


def test_selective_refuses():
    lib = ssd.raw()
    need = ssd.selective_prefill_workspace_bytes(shape())
    assert need > 0 and need % 256 == 0
    T = ssd.ssd_dt_transform

    def prefill(s=shape(), x=FAKE, dt=FAKE, A=FAKE, B=FAKE, bs=16, C=FAKE, cs=16, D=FAKE, z=FAKE, zs=96, cu=FAKE, h0=FAKE, y=FAKE, f=FAKE, w=FAKE,
                wb=need, tr=T(4096, 1, 0.0, 0.0)):
        return lib.ssd_selective_prefill(None if s is None else ctypes.byref(s), None if tr is None else ctypes.byref(tr), cu, x, dt, A, B, bs, C, cs, D,
                                         z, zs, h0, y, f, w, ctypes.c_size_t(wb), None)

    def step(s=shape(), x=FAKE, dt=FAKE, A=FAKE, B=FAKE, bs=16, C=FAKE, cs=16, D=FAKE, z=FAKE, zs=96, f=FAKE, y=FAKE, tr=T(4096, 1, 0.0, 0.0), wb=None):
        return lib.ssd_selective_step(None if s is None else ctypes.byref(s), None if tr is None else ctypes.byref(tr), f, x, dt, A, B, bs, C, cs, D, z, zs,
                                      y, None)

    for f in (prefill, step):
        assert f(s=None) == -1
        for bad, status in BAD:
            assert f(s=shape(**bad), wb=1 << 60) == status, bad
            assert ssd.selective_prefill_workspace_bytes(shape(**bad)) == 0
        refusals(f, ("x", "dt", "A", "B", "C", "y", "f"), ("x", "dt", "A", "D", "y", "f"), ("B", "C", "z"))
        assert f(bs=15) == -2 and f(cs=15) == -2 and f(zs=95) == -2 and f(bs=1 << 60) == -4 and f(zs=(1 << 24) + 1) == -4
        assert f(tr=T(4100, 1, 0.0, 0.0)) == -7 and f(tr=T(4096, 1, 0.2, 0.1)) == -2 and f(tr=T(4096, 1, float("nan"), 0.1)) == -2
        assert f(s=shape(io_dtype=0, dt_dtype=0), B=HALF, wb=1 << 60) == -7
    refusals(prefill, ("cu",), ("h0",), ("cu",))
    assert prefill(s=shape(tokens=0)) == -2 and prefill(s=shape(tokens=(1 << 30) + 1)) == -2 and prefill(s=shape(tokens=1 << 30, dstate=256)) == -2
    assert prefill(w=None) == -5 and prefill(wb=need - 1) == -5 and prefill(w=ctypes.c_void_p(4096 + 16)) == -5


def test_workspace_grows_with_the_tokens():
    for channels, dstate in ((64, 16), (1536, 16), (5120, 16), (100, 7), (768, 256)):
        last = 0
        for tokens in list(range(1, 2000, 37)) + [4096, 4097, 16384, 100000, 1 << 20]:
            need = ssd.selective_prefill_workspace_bytes(shape(tokens=tokens, channels=channels, dstate=dstate))
            assert need >= last, (channels, dstate, tokens)
            last = need


ATTN = dict(batch=3, tokens=20, nheads=8, nkvheads=2, headdim=64, npages=100, page_size=16, max_pages=10, window=0, io_dtype=1)


def test_append_norm_refuses():
    lib = ssd.raw()

    def call(s=ssd.ssd_attn_shape(**ATTN), rope=(4096, 4096, 64, 160, 0), cu=FAKE, lens=FAKE, table=FAKE, q=FAKE, qs=512, k=FAKE, ks=128, v=FAKE, vs=128,
             qw=FAKE, kw=FAKE, eps=1e-5, qo=ctypes.c_void_p(1 << 20), kc=FAKE, vc=FAKE):
        r = None if rope is None else ctypes.byref(ssd.ssd_rope(*rope))
        return lib.ssd_attn_append_norm(None if s is None else ctypes.byref(s), r, cu, lens, table, q, qs, k, ks, v, vs, qw, kw, eps, qo, kc, vc, None)

    assert call(s=None) == -1 and call(rope=None) == -1
    for bad, status in ((dict(batch=0), -2), (dict(nkvheads=3), -2), (dict(headdim=60), -4), (dict(headdim=264), -4), (dict(page_size=24), -4),
                        (dict(io_dtype=2), -3), (dict(tokens=0), -2)):
        assert call(s=ssd.ssd_attn_shape(**dict(ATTN, **bad))) == status, bad
    assert call(eps=-1e-5) == -2 and call(eps=float("nan")) == -2
    refusals(call, ("lens", "table", "k", "v", "kc", "vc", "q", "qo", "qw", "kw"), ("k", "v", "kc", "vc", "q", "qo", "qw", "kw"), ("cu", "lens", "table"))
    assert call(rope=(4096, 4096, 63, 160, 0)) == -2 and call(rope=(4096, 4096, 64, 159, 0)) == -2 and call(rope=(4096, 0, 64, 160, 0)) == -1
    assert call(qs=511) == -2 and call(ks=129) == -7
    assert call(qo=FAKE) == -4, "rotated queries over their inputs"


def test_binding_refuses():
    t = lambda *s, dt=torch.bfloat16: torch.zeros(s, dtype=dt)   # noqa: E731
    f, i = torch.float32, torch.int32
    cu = torch.tensor([0, 3, 5], dtype=i)
    conv = dict(u=t(5, 12), weight=t(12, 4, dt=f), bias=t(12, dt=f), cu_seqlens=cu, conv_state=t(2, 12, 3))
    for bad in ({}, dict(u=t(5, 11)), dict(weight=t(12, 4)), dict(cu_seqlens=cu.long()), dict(cu_seqlens=cu[:1]), dict(conv_state=t(1, 12, 3)),
                dict(conv_state=t(2, 12, 3, dt=f)), dict(split=(8, 8)), dict(outs=[]), dict(outs=[t(5, 12, dt=f)]), dict(outs=[t(4, 12)]),
                dict(conv_state_out=t(2, 12, 2)), dict(u=t(5, 1).expand(5, 12)), dict(u=t(1, 12).expand(5, 12)), dict(bias=t(12))):
        with pytest.raises(ValueError):
            ssd.ssd_conv1d_varlen(**dict(conv, **bad))
    both = dict(x=t(5, 12), dt=t(5, 12), A=t(12, 4, dt=f), B=t(5, 4), C=t(5, 4), D=t(12, dt=f), z=t(5, 12), dt_bias=t(12, dt=f))
    bads = ({}, dict(dt=t(5, 11)), dict(A=t(12, 4)), dict(A=t(11, 4, dt=f)), dict(B=t(5, 3)), dict(C=t(4, 4)), dict(B=t(5, 4, dt=f)), dict(D=t(12)),
            dict(z=t(5, 11)), dict(z=t(5, 12, dt=f)), dict(z=t(1, 12).expand(5, 12)), dict(dt_bias=t(11, dt=f)), dict(y=t(5, 11)), dict(y=t(5, 12, dt=f)),
            dict(dt=t(5, 12, dt=torch.float16)))
    for bad in bads + (dict(cu_seqlens=cu.long()), dict(h0=t(1, 12, 4, dt=f)), dict(h0=t(2, 12, 4)), dict(final_state=t(1, 12, 4, dt=f))):
        with pytest.raises((ValueError, ssd.SSDError)):
            ssd.ssd_selective_prefill(**dict(both, cu_seqlens=cu, **bad) if "cu_seqlens" not in bad else dict(both, **bad))
    for bad in bads + (dict(state=t(5, 12, 3, dt=f)), dict(state=t(5, 12, 4))):
        with pytest.raises((ValueError, ssd.SSDError)):
            ssd.ssd_selective_step(**dict(dict(both, state=t(5, 12, 4, dt=f)), **bad))
    app = dict(q=t(5, 4, 8), k=t(5, 2, 8), v=t(5, 2, 8), q_weight=t(8, dt=f), k_weight=t(8, dt=f), k_cache=t(3, 2, 16, 8), v_cache=t(3, 2, 16, 8),
               page_table=t(2, 2, dt=i), seq_lens=t(2, dt=i), cu_seqlens=cu)
    for bad in ({}, dict(q_weight=None), dict(q=None), dict(k_weight=t(8)), dict(k_weight=t(4, dt=f)), dict(v=t(5, 2, 4)), dict(cu_seqlens=None)):
        with pytest.raises((ValueError, AttributeError)):
            ssd.ssd_attn_append_norm(**dict(app, **bad))
