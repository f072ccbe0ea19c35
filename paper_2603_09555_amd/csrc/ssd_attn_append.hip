// Appends new tokens' keys and values to a paged cache; queries and keys are rotated by their positions on the way.
//
//   position of new token j of sequence b:  p = seq_lens[b] - (new tokens of b) + j
//   pair (a, c) of head values:             (a cos - c sin, c cos + a sin),  cos, sin = rope[p][pair]
//   key, value  ->  page table[b][p / page_size], slot p % page_size
//
// A copy in effect: each value is read and written once, bound by memory, or by the chain of memory latencies for few tokens
// (boundaries, length, page, then the values).  A workgroup finds the places of a few neighbouring tokens once; its threads then
// take their pieces of 16 bytes in turn.  A piece that holds one half of its pairs brings the other halves' piece with it, which
// its neighbour brings too, from the first-level cache.
// 12 prompts of 1 to 5119 tokens, 40 heads over 8 of 64, bf16: 57 us, 4.1 TB/s, fp32: 98 us, 4.8; 64 single tokens, 32 heads over 8 of
// 128: 4.3 us, fp32 the same.
#include <algorithm>

#include "ssd_attn.hpp"

namespace ssd {
namespace {

using namespace block;

constexpr int kBatch = 2;        // tokens whose pieces a thread has on their way at a time
constexpr int kMostTokens = 4;   // a workgroup
constexpr int kFewWorkgroups = 2048;  // more take several tokens each

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
  int run;                 // tokens a workgroup
};

struct Place {
  int pos;       // < 0: none
  int64_t slot;  // cache row of key head 0, or -1
};

template <bool kBf16>
using Element = typename std::conditional<kBf16, uint16_t, float>::type;
__device__ __forceinline__ float value(float v) { return v; }
__device__ __forceinline__ float value(uint16_t v) { return __uint_as_float(static_cast<uint32_t>(v) << 16); }
template <bool kBf16, int W>
__device__ __forceinline__ void unpack(const u32x4 &q, float (&v)[W]) {
#pragma unroll
  for (int i = 0; i < W; ++i) v[i] = !kBf16 ? __uint_as_float(q[i % 4]) : i % 2 == 0 ? bf_lo(q[i / 2]) : bf_hi(q[i / 2]);
}
// N neighbouring values at an address of any multiple of 4
template <int N>
__device__ __forceinline__ void load_rope(const float *p, float *v) {
  typedef f32x4 __attribute__((aligned(4))) vec4;
  typedef float f32x2 __attribute__((ext_vector_type(2)));
  typedef f32x2 __attribute__((aligned(4))) vec2;
  if constexpr (N == 2) {
    const f32x2 a = *reinterpret_cast<const vec2 *>(p);
    v[0] = a[0];
    v[1] = a[1];
  } else {
#pragma unroll
    for (int i = 0; i < N; i += 4) {
      const f32x4 a = *reinterpret_cast<const vec4 *>(p + i);
#pragma unroll
      for (int k = 0; k < 4; ++k) v[i + k] = a[k];
    }
  }
}

// kWhole: pieces lie in one half of the pairs (interleaved pairs: in the rotated part) or outside it.
template <bool kBf16, bool kWhole>
__global__ __launch_bounds__(256) void append_kernel(const AppendArgs a) {
  using E = Element<kBf16>;
  constexpr int W = 16 / sizeof(E);
  __shared__ Place place[kMostTokens];
  const int first_token = blockIdx.x * a.run, tokens = min(a.run, a.d.T - first_token);
  if (static_cast<int>(threadIdx.x) < tokens) {
    const Token t = find_token(a.d, a.cu, a.lens, first_token + threadIdx.x);
    place[threadIdx.x] = {t.pos, t.pos < 0 ? -1 : slot_of(a.d, a.table, t.seq, t.pos, 0)};
  }
  __syncthreads();
  // this thread's piece of a token: which of q, k, v, its head and first value
  const int idx = blockIdx.y * 256 + threadIdx.x;
  if (idx >= a.row_pieces) return;
  int head = quotient(idx, a.head_pieces, a.inv_head_pieces), what = 0;
  const int first = (idx - head * a.head_pieces) * W;
  if (head >= a.q_heads) {
    head -= a.q_heads;
    what = 1;
    if (head >= a.d.Hk) {
      head -= a.d.Hk;
      what = 2;
    }
  }
  const int64_t stride = a.stride[what];
  const E *const src = static_cast<const E *>(a.src[what]) + first_token * stride + static_cast<int64_t>(head) * a.d.D;
  E *const out = what == 0 ? static_cast<E *>(a.q_out) + (static_cast<int64_t>(first_token) * a.d.H + head) * a.d.D + first
                           : static_cast<E *>(a.cache[what - 1]) + (static_cast<int64_t>(head) << a.d.lg_page) * a.d.D + first;
  const int64_t out_stride = static_cast<int64_t>(a.d.H) * a.d.D;
  const int half = a.rope.half;
  const bool rotated = what < 2 && first < 2 * half, second = !a.rope.interleaved && first >= half;
  const int partner = second ? first - half : first + half, pair = a.rope.interleaved ? first / 2 : second ? first - half : first;
  // kBatch tokens at a time: asked for together, then written
  for (int token0 = 0; token0 < tokens; token0 += kBatch) {
    u32x4 q[kBatch], other[kBatch];
    Place at[kBatch];
#pragma unroll
    for (int k = 0; k < kBatch; ++k) {
      at[k].pos = -1;
      if (token0 + k >= tokens) continue;
      at[k] = place[token0 + k];
      if (at[k].pos < 0 || (what > 0 && at[k].slot < 0)) {
        at[k].pos = -1;
        continue;
      }
      const E *const row = src + (token0 + k) * stride;
      q[k] = *reinterpret_cast<const u32x4 *>(row + first);
      if (kWhole && rotated && !a.rope.interleaved) other[k] = *reinterpret_cast<const u32x4 *>(row + partner);
    }
#pragma unroll
    for (int k = 0; k < kBatch; ++k) {
      if (at[k].pos < 0) continue;
      if (rotated) {
        const float *const cs = a.rope.cos + static_cast<int64_t>(at[k].pos) * half, *const sn = a.rope.sin + static_cast<int64_t>(at[k].pos) * half;
        float v[W], r[W];
        unpack<kBf16>(q[k], v);
        if (kWhole && !a.rope.interleaved) {
          float o[W], c[W], s[W];
          unpack<kBf16>(other[k], o);
          load_rope<W>(cs + pair, c);
          load_rope<W>(sn + pair, s);
#pragma unroll
          for (int i = 0; i < W; ++i) r[i] = fmaf(v[i], c[i], second ? o[i] * s[i] : -o[i] * s[i]);
        } else if (kWhole) {
          float c[W / 2], s[W / 2];
          load_rope<W / 2>(cs + pair, c);
          load_rope<W / 2>(sn + pair, s);
#pragma unroll
          for (int i = 0; i < W; i += 2) {
            r[i] = fmaf(v[i], c[i / 2], -v[i + 1] * s[i / 2]);
            r[i + 1] = fmaf(v[i + 1], c[i / 2], v[i] * s[i / 2]);
          }
        } else {
          const E *const row = src + (token0 + k) * stride;
#pragma unroll
          for (int i = 0; i < W; ++i) {
            const int c = first + i;
            r[i] = v[i];
            if (c < 2 * half) {
              const bool b = a.rope.interleaved ? (c & 1) : c >= half;  // the second of its pair
              const int p = a.rope.interleaved ? c >> 1 : b ? c - half : c;
              const float o = value(row[a.rope.interleaved ? c ^ 1 : b ? c - half : c + half]);
              r[i] = fmaf(v[i], cs[p], b ? o * sn[p] : -o * sn[p]);
            }
          }
        }
        if constexpr (kBf16) {
#pragma unroll
          for (int i = 0; i < 4; ++i) q[k][i] = pack2(r[2 * i], r[2 * i + 1]);
        } else {
#pragma unroll
          for (int i = 0; i < 4; ++i) q[k][i] = __float_as_uint(r[i]);
        }
      }
      *reinterpret_cast<u32x4 *>(out + (what == 0 ? (token0 + k) * out_stride : at[k].slot * a.d.D)) = q[k];
    }
  }
}

}  // namespace

namespace {

int row_pieces(const AttnDims &d, bool queries) { return ((queries ? d.H : 0) + 2 * d.Hk) * (d.D / (d.bf16 ? 8 : 4)); }
int parts_of(int pieces) { return (pieces + 255) / 256; }
int run_of(const AttnDims &d, int parts) {
  return static_cast<int>(std::max<int64_t>(1, std::min<int64_t>(kMostTokens, static_cast<int64_t>(d.T) * parts / kFewWorkgroups)));
}

}  // namespace

bool attn_append_fits(const AttnDims &d, bool queries) {
  const int run = run_of(d, parts_of(row_pieces(d, queries)));
  return (static_cast<int64_t>(d.T) + run - 1) / run <= kMostWorkgroups256;
}

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
  a.row_pieces = row_pieces(d, q != nullptr);
  const int parts = parts_of(a.row_pieces);
  a.run = run_of(d, parts);
  const dim3 grid((d.T + a.run - 1) / a.run, parts);
  const int width = rope.interleaved ? 2 * rope.half : rope.half;
  const bool whole = width % (d.bf16 ? 8 : 4) == 0;
  if (d.bf16 && whole)
    hipLaunchKernelGGL((append_kernel<true, true>), grid, dim3(256), 0, stream, a);
  else if (d.bf16)
    hipLaunchKernelGGL((append_kernel<true, false>), grid, dim3(256), 0, stream, a);
  else if (whole)
    hipLaunchKernelGGL((append_kernel<false, true>), grid, dim3(256), 0, stream, a);
  else
    hipLaunchKernelGGL((append_kernel<false, false>), grid, dim3(256), 0, stream, a);
  return hipGetLastError();
}

}  // namespace ssd
