"""What the norms and the operators on a paged cache refuse, before any HIP call (so these run on a CPU machine): through the C
ABI, and through the Python binding on tensors that are never looked into."""
import ctypes

import pytest
import torch

from paper_2603_09555_amd import ssd

FAKE = ctypes.c_void_p(4096)   # never dereferenced: validation fails first
OK = dict(batch=3, tokens=20, nheads=8, nkvheads=2, headdim=64, npages=100, page_size=16, max_pages=10, window=0, io_dtype=1)
BAD_SHAPES = [(dict(batch=0), -2), (dict(nheads=0), -2), (dict(nkvheads=3), -2), (dict(nkvheads=0), -2), (dict(headdim=0), -2),
              (dict(npages=0), -2), (dict(page_size=0), -2), (dict(max_pages=0), -2), (dict(window=-1), -2), (dict(io_dtype=2), -3),
              (dict(headdim=264), -4), (dict(headdim=60), -4), (dict(page_size=24), -4), (dict(page_size=1 << 17), -4),
              (dict(nheads=65536, nkvheads=65536), -4), (dict(max_pages=1 << 30), -2), (dict(npages=2 ** 31 - 1, page_size=65536, max_pages=1), -2)]


def shape(**kw):
    return ssd.ssd_attn_shape(**dict(OK, **kw))


def test_attention_refuses():
    lib = ssd.raw()
    need_s, need_p = ssd.attn_step_workspace_bytes(shape()), ssd.attn_prefill_workspace_bytes(shape())
    assert need_s > 0 and need_p > 0 and need_s % 256 == 0 and need_p % 256 == 0

    def step(s=shape(), lens=FAKE, table=FAKE, q=FAKE, k=FAKE, v=FAKE, y=FAKE, w=FAKE, wb=need_s, scale=0.1):
        return lib.ssd_attn_step(ctypes.byref(s) if s is not None else None, lens, table, q, k, v, scale, y, w, ctypes.c_size_t(wb), None)

    def prefill(s=shape(), lens=FAKE, table=FAKE, q=FAKE, k=FAKE, v=FAKE, y=FAKE, w=FAKE, wb=need_p, cu=FAKE, scale=0.1):
        return lib.ssd_attn_prefill(ctypes.byref(s) if s is not None else None, cu, lens, table, q, k, v, scale, y, w, ctypes.c_size_t(wb), None)

    odd, half = ctypes.c_void_p(4104), ctypes.c_void_p(4098)
    for f, need in ((step, need_s), (prefill, need_p)):
        assert f(s=None) == -1
        for bad, status in BAD_SHAPES:
            assert f(s=shape(**bad), wb=1 << 50) == status, bad
            assert ssd.attn_step_workspace_bytes(shape(**bad)) == 0 and ssd.attn_prefill_workspace_bytes(shape(**bad)) == 0
        for name in ("lens", "table", "q", "k", "v", "y"):
            assert f(**{name: None}) == -1, name
            assert f(**{name: half if name in ("lens", "table") else odd}) == -7, name
        assert f(scale=0.0) == -2 and f(scale=-1.0) == -2 and f(scale=float("nan")) == -2 and f(scale=float("inf")) == -2
        assert f(w=None) == -5 and f(wb=need - 1) == -5 and f(w=ctypes.c_void_p(4096 + 16)) == -5
    assert prefill(cu=None) == -1 and prefill(cu=half) == -7 and prefill(s=shape(tokens=0)) == -2
    assert ssd.attn_step_workspace_bytes(shape(tokens=0)) == need_s   # (the step ignores tokens)


def test_append_refuses():
    lib = ssd.raw()

    def call(s=shape(), rope=(FAKE, FAKE, 64, 160, 0), cu=FAKE, lens=FAKE, table=FAKE, q=FAKE, qs=512, k=FAKE, ks=128, v=FAKE, vs=128, qo=FAKE,
             kc=FAKE, vc=FAKE):
        r = None if rope is None else ctypes.byref(ssd.ssd_rope(*[x.value if isinstance(x, ctypes.c_void_p) else x for x in rope]))
        return lib.ssd_attn_append(ctypes.byref(s) if s is not None else None, r, cu, lens, table, q, qs, k, ks, v, vs, qo, kc, vc, None)

    assert call(s=None) == -1 and call(rope=None) == -1
    for bad, status in BAD_SHAPES:
        assert call(s=shape(**bad)) == status, bad
    assert call(s=shape(tokens=0)) == -2
    for name in ("lens", "table", "k", "v", "kc", "vc", "q", "qo"):   # (q and q_out: one without the other)
        assert call(**{name: None}) == -1, name
        assert call(**{name: ctypes.c_void_p(4098)}) == -7, name
    assert call(cu=ctypes.c_void_p(4098)) == -7
    assert call(rope=(None, FAKE, 64, 160, 0)) == -1 and call(rope=(FAKE, ctypes.c_void_p(4100), 64, 160, 0)) == -7
    assert call(rope=(FAKE, FAKE, 63, 160, 0)) == -2 and call(rope=(FAKE, FAKE, 66, 160, 0)) == -2 and call(rope=(FAKE, FAKE, -2, 160, 0)) == -2
    assert call(rope=(FAKE, FAKE, 64, 159, 0)) == -2, "a row for every position the page table can hold"
    assert call(rope=(FAKE, FAKE, 64, 160, 2)) == -2
    assert call(qs=511) == -2 and call(ks=127) == -2 and call(vs=64) == -2
    assert call(qs=516) == -7 and call(ks=129) == -7 and call(vs=130) == -7


def test_norms_refuse():
    lib = ssd.raw()

    def gated(rows=4, width=64, groups=1, io=1, y=FAKE, z=FAKE, zs=64, w=FAKE, eps=1e-5, first=0, out=FAKE):
        return lib.ssd_norm_gated(rows, width, groups, io, y, z, zs, w, eps, first, out, None)

    def residual(rows=4, width=64, io=1, rio=0, x=FAKE, r=FAKE, w=FAKE, eps=1e-5, out=FAKE, ro=FAKE):
        return lib.ssd_norm_residual(rows, width, io, rio, x, r, 1.0, w, eps, out, ro, None)

    for f in (gated, residual):
        assert f(rows=0) == -2 and f(width=0) == -2 and f(eps=-1.0) == -2 and f(eps=float("nan")) == -2 and f(rows=1 << 40) == -2
        assert f(io=2) == -3 and f(w=None) == -1 and f(out=None) == -1
        assert f(w=ctypes.c_void_p(4100)) == -7 and f(out=ctypes.c_void_p(4104)) == -7
    assert gated(groups=3) == -2 and gated(groups=0) == -2 and gated(zs=63) == -2 and gated(first=2) == -2
    assert gated(y=None) == -1 and gated(z=None) == -1 and gated(y=ctypes.c_void_p(4098)) == -7 and gated(z=ctypes.c_void_p(4097)) == -7
    assert gated(io=0, z=ctypes.c_void_p(4098)) == -7
    assert residual(rio=2) == -3 and residual(io=0, rio=1) == -3 and residual(x=None) == -1 and residual(ro=None) == -1
    assert residual(r=ctypes.c_void_p(4104)) == -7 and residual(ro=ctypes.c_void_p(4104)) == -7 and residual(x=ctypes.c_void_p(4104)) == -7


def test_the_binding_refuses():
    q, kv, cache = torch.zeros(3, 8, 64), torch.zeros(3, 2, 64), torch.zeros(5, 2, 16, 64)
    table, lens, cu = torch.zeros(3, 4, dtype=torch.int32), torch.zeros(3, dtype=torch.int32), torch.zeros(4, dtype=torch.int32)
    for call, match in (
            (lambda: ssd.ssd_attn_step(q.bfloat16(), cache, cache, table, lens), "one dtype"),
            (lambda: ssd.ssd_attn_step(q, cache, cache, table.long(), lens), "int32"),
            (lambda: ssd.ssd_attn_step(q, cache, cache[:4], table, lens), "shapes"),
            (lambda: ssd.ssd_attn_step(q, cache, cache, table, lens[:2]), "shapes"),
            (lambda: ssd.ssd_attn_step(q[:, :, :32], cache, cache, table, lens), "shapes"),
            (lambda: ssd.ssd_attn_step(q, cache, cache, table, lens), "device tensors"),
            (lambda: ssd.ssd_attn_prefill(q, cache, cache, table, lens, None), "cu_seqlens"),
            (lambda: ssd.ssd_attn_prefill(q, cache, cache, table, lens, cu[:3]), "shapes"),
            (lambda: ssd.ssd_attn_append(q, kv, kv.bfloat16(), cache, cache, table, lens), "one dtype"),
            (lambda: ssd.ssd_attn_append(q[:2], kv, kv, cache, cache, table, lens), "agree"),
            (lambda: ssd.ssd_attn_append(q, kv, kv, cache, cache, table, lens), "device tensors"),
            (lambda: ssd.ssd_norm_gated(kv[0], kv[0, :1], torch.zeros(64)), "like y"),
            (lambda: ssd.ssd_norm_gated(kv[0], kv[0], torch.zeros(64).bfloat16()), "weight"),
            (lambda: ssd.ssd_norm_gated(kv[0], kv[0], torch.zeros(64)), "device tensor"),
            (lambda: ssd.ssd_norm_residual(kv[0, :1], kv[0], torch.zeros(64)), "shape of x"),
            (lambda: ssd.ssd_norm_residual(None, kv[0], torch.zeros(64), out=torch.zeros(2)), "too small"),
            (lambda: ssd.ssd_norm_residual(None, kv[0], torch.zeros(64)), "device tensors")):
        with pytest.raises(ValueError, match=match):
            call()
