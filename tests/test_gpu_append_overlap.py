"""A thread that rotates reads values that another one writes: q_out must not reach into q, k or v."""
import ctypes

import pytest
import torch

from paper_2603_09555_amd import ssd

H, HK, D, T = 4, 2, 64, 20


def append(base, q, k, v, q_out, stride, tokens=T, dtype=1):
    """The C call with tensors at these bytes behind ``base``.  (Nothing here is looked into: each call is refused.)"""
    size = 2 if dtype == 1 else 4
    s, rope = ssd.ssd_attn_shape(1, tokens, H, HK, D, 100, 16, 10, 0, dtype), ssd.ssd_rope(None, None, 0, 0, 0)
    at = [ctypes.c_void_p(base + o) for o in (q, k, v, q_out)]
    n, fake = ctypes.c_int64(stride // size), ctypes.c_void_p(4096)
    return ssd.raw().ssd_attn_append(ctypes.byref(s), ctypes.byref(rope), fake, fake, fake, at[0], n, at[1], n, at[2], n, at[3], fake, fake, None)


@pytest.mark.parametrize("dtype", [0, 1])
def test_refused(dtype):
    size = 2 if dtype == 1 else 4
    head = D * size
    row, stride = H * head, (H + 2 * HK) * head      # one projection's output: queries, keys, values
    k, v, far = row, row + HK * head, 1 << 20
    base = 1 << 30
    for q_out in (0, 16, -row, -(T * row) + 16, stride, k, v, v + HK * head - 16, (T - 1) * stride, T * stride - 16):
        assert append(base, 0, k, v, q_out, stride, dtype=dtype) == -4, q_out
    # dense tensors, one of which it reaches into; and a gap between two rows that is too small
    for at in range(3):
        where = [4 * far, 5 * far, 6 * far]
        where[at] = 0
        assert append(base, *where, T * row - 16 if at == 0 else 0, row, dtype=dtype) == -4, at
    assert append(base, 0, far, 2 * far, row, 2 * row, tokens=2, dtype=dtype) == -4


@pytest.mark.gpu
@pytest.mark.parametrize("io", [torch.float32, torch.bfloat16], ids=str)
def test_taken_and_refused_on_tensors(io):
    g = torch.Generator(device="cuda").manual_seed(1)
    cache, table = torch.zeros(3, HK, 16, D, device="cuda", dtype=io), torch.tensor([[0, 1, 2]], dtype=torch.int32, device="cuda")
    lens, cu = torch.tensor([T], dtype=torch.int32, device="cuda"), torch.tensor([0, T], dtype=torch.int32, device="cuda")
    rope = [torch.randn(48, D // 2, generator=g, device="cuda") for _ in range(2)]
    args = (cache, cache.clone(), table, lens, cu)
    qkv = torch.randn(T, H + 2 * HK, D, generator=g, device="cuda").to(io)
    q, k, v = qkv.split((H, HK, HK), dim=1)
    ref = ssd.ssd_attn_append(q, k, v, *args, rope=rope)
    dense = q.contiguous()
    for q_in, out in ((dense, dense), (q, qkv.view(-1)[:T * H * D].view(T, H, D)), (dense, torch.empty(T + 1, H, D, device="cuda", dtype=io)[1:])):
        clash = out.data_ptr() in (q_in.data_ptr(), qkv.data_ptr())
        if clash:
            with pytest.raises(ssd.SSDError) as e:
                ssd.ssd_attn_append(q_in, k, v, *args, rope=rope, q_out=out)
            assert e.value.status == -4
        else:
            assert torch.equal(ssd.ssd_attn_append(q_in, k, v, *args, rope=rope, q_out=out), ref)
    # right behind q, right in front of it, and between two rows of it
    room = torch.randn(3 * T, H, D, generator=g, device="cuda").to(io)
    room[T:2 * T] = q
    for out in (room[2 * T:], room[:T]):
        assert torch.equal(ssd.ssd_attn_append(room[T:2 * T], k, v, *args, rope=rope, q_out=out), ref)
    wide = torch.randn(2, 4 * H, D, generator=g, device="cuda").to(io)
    two = (cache, cache.clone(), table, lens, torch.tensor([0, 2], dtype=torch.int32, device="cuda"))
    ref = ssd.ssd_attn_append(wide[:, :H], k[:2], v[:2], *two, rope=rope)
    out = wide.view(-1)[H * D:3 * H * D].view(2, H, D)
    assert torch.equal(ssd.ssd_attn_append(wide[:, :H], k[:2], v[:2], *two, rope=rope, q_out=out), ref)
