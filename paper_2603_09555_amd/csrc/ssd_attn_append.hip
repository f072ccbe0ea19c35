// Appends new tokens' keys and values to a paged cache; queries and keys are rotated by their positions on the way.
//
//   position of new token j of sequence b:  p = seq_lens[b] - (new tokens of b) + j
//   pair (a, c) of head values:             (a cos - c sin, c cos + a sin),  cos, sin = rope[p][pair]
//   key, value  ->  page table[b][p / page_size], slot p % page_size
//
// A copy in effect: each value is read and written once.  A thread writes one piece of 16 bytes of one head of one token
// (and reads the piece that holds the other halves of its pairs, which a neighbour reads too, from the first-level cache).
#include "ssd_attn.hpp"

namespace ssd {
namespace {

using namespace block;

struct AppendArgs {
  const void *src[3];      // q, k, v
  int64_t stride[3];
  void *q_out, *cache[2];
  const int32_t *cu, *lens, *table;
  AttnDims d;
  Rope rope;
  int head_pieces;         // pieces of a head
  uint32_t inv_head_pieces;
  int row_pieces;          // pieces of a token: queries (if any), keys, values
  int q_heads;             // 0: no queries
};

template <typename E>
__device__ __forceinline__ float value(E v);
template <>
__device__ __forceinline__ float value<float>(float v) { return v; }
template <>
__device__ __forceinline__ float value<uint16_t>(uint16_t v) { return __uint_as_float(static_cast<uint32_t>(v) << 16); }

template <bool kBf16>
__global__ __launch_bounds__(256) void append_kernel(const AppendArgs a) {
  using E = typename std::conditional<kBf16, uint16_t, float>::type;
  constexpr int W = 16 / sizeof(E);
  const int token = blockIdx.x;
  const int idx = blockIdx.y * 256 + threadIdx.x;
  const Token at = find_token(a.d, a.cu, a.lens, token);
  if (!at.found || at.pos < 0 || idx >= a.row_pieces) return;
  int head = quotient(idx, a.head_pieces, a.inv_head_pieces);
  const int first = (idx - head * a.head_pieces) * W;
  // which of q, k, v
  int what = 0;
  if (head >= a.q_heads) {
    head -= a.q_heads;
    what = 1;
    if (head >= a.d.Hk) {
      head -= a.d.Hk;
      what = 2;
    }
  }
  E *dst;
  if (what == 0) {
    dst = static_cast<E *>(a.q_out) + (static_cast<int64_t>(token) * a.d.H + head) * a.d.D + first;
  } else {
    const int64_t slot = slot_of(a.d, a.table, at.seq, at.pos, head);
    if (slot < 0) return;
    dst = static_cast<E *>(a.cache[what - 1]) + slot * a.d.D + first;
  }
  const E *src = static_cast<const E *>(a.src[what]) + token * a.stride[what] + static_cast<int64_t>(head) * a.d.D;
  u32x4 q = *reinterpret_cast<const u32x4 *>(src + first);
  const int half = a.rope.half;
  if (what < 2 && first < 2 * half) {
    const float *cs = a.rope.cos + static_cast<int64_t>(at.pos) * half, *sn = a.rope.sin + static_cast<int64_t>(at.pos) * half;
    E e[W];
    __builtin_memcpy(e, &q, 16);
    float r[W];
#pragma unroll
    for (int i = 0; i < W; ++i) {
      const int c = first + i;
      r[i] = value(e[i]);
      if (c < 2 * half) {
        const bool second = a.rope.interleaved ? (c & 1) : c >= half;
        const int pair = a.rope.interleaved ? c >> 1 : second ? c - half : c;
        const int other = a.rope.interleaved ? c ^ 1 : second ? c - half : c + half;
        const float o = value(src[other]);
        r[i] = fmaf(r[i], cs[pair], second ? o * sn[pair] : -o * sn[pair]);
      }
    }
    if (kBf16) {
#pragma unroll
      for (int i = 0; i < 4; ++i) q[i] = pack2(r[(2 * i) % W], r[(2 * i + 1) % W]);
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) q[i] = __float_as_uint(r[i]);
    }
  }
  *reinterpret_cast<u32x4 *>(dst) = q;
}

}  // namespace

hipError_t launch_attn_append(const AttnDims &d, const Rope &rope, const int32_t *cu, const int32_t *lens, const int32_t *table,
                              const void *q, int64_t q_stride, const void *k, int64_t k_stride, const void *v, int64_t v_stride,
                              void *q_out, void *k_cache, void *v_cache, hipStream_t stream) {
  AppendArgs a = {};
  a.src[0] = q;
  a.src[1] = k;
  a.src[2] = v;
  a.stride[0] = q_stride;
  a.stride[1] = k_stride;
  a.stride[2] = v_stride;
  a.q_out = q_out;
  a.cache[0] = k_cache;
  a.cache[1] = v_cache;
  a.cu = cu;
  a.lens = lens;
  a.table = table;
  a.d = d;
  a.rope = rope;
  a.q_heads = q != nullptr ? d.H : 0;
  a.head_pieces = d.D / (d.bf16 ? 8 : 4);
  a.inv_head_pieces = inverse_of(a.head_pieces);
  a.row_pieces = (a.q_heads + 2 * d.Hk) * a.head_pieces;
  const dim3 grid(d.T, (a.row_pieces + 255) / 256);
  if (d.bf16)
    hipLaunchKernelGGL(append_kernel<true>, grid, dim3(256), 0, stream, a);
  else
    hipLaunchKernelGGL(append_kernel<false>, grid, dim3(256), 0, stream, a);
  return hipGetLastError();
}

}  // namespace ssd
