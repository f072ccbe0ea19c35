// Appends new tokens' keys and values to a paged cache; heads of queries and keys are normalised and rotated by their positions
// on the way:
//
//   u = v rsqrt(mean(v^2) + eps) weight        over the headdim values of a head
//   pair (a, c) of u:  (a cos - c sin, c cos + a sin),  cos, sin = rope[p][pair],  p = seq_lens[b] - (new tokens of b) + j
//   key, value  ->  page table[b][p / page_size], slot p % page_size;  rounded once
//
// A copy in effect, like the append without norms.  A head is held by as many neighbouring lanes as it has pieces of 16 bytes
// (rounded up to a power of two), so that the sum of its squares stays within a wave; a thread's piece of the head vector, and
// with it its weights, are the same for all its tokens.  A piece that holds one half of its pairs brings the other halves'
// piece with it, which a lane nearby brings too, from the first-level cache.
#include <algorithm>

#include "ssd_attn_append.hpp"

namespace ssd {
namespace {

struct AppendNormArgs {
  const void *src[3];      // q, k, v
  int64_t stride[3];
  const float *weight[2];  // of queries, of keys
  void *q_out, *cache[2];
  const int32_t *cu, *lens, *table;
  AttnDims d;
  Rope rope;
  float eps, inv_headdim;
  int lg_lanes;            // lanes a head: 2^lg_lanes
  int q_heads;             // 0: no queries
  int run;                 // tokens a workgroup
};

// kWhole: pieces lie in one half of the pairs (interleaved pairs: in the rotated part) or outside it.
template <bool kBf16, bool kWhole>
__global__ __launch_bounds__(256) void append_norm_kernel(const AppendNormArgs a) {
  using E = Element<kBf16>;
  constexpr int W = 16 / sizeof(E);
  __shared__ Place place[kMostTokens];
  const int first_token = blockIdx.x * a.run, tokens = min(a.run, a.d.T - first_token);
  if (static_cast<int>(threadIdx.x) < tokens) {
    const Token t = find_token(a.d, a.cu, a.lens, first_token + threadIdx.x);
    place[threadIdx.x] = {t.pos, t.pos < 0 ? -1 : slot_of(a.d, a.table, t.seq, t.pos, 0)};
  }
  __syncthreads();
  // this thread's head -- of q, k or v -- and its piece's first value; lanes of a head enter and leave together
  const int lanes = 1 << a.lg_lanes;
  int head = static_cast<int>((blockIdx.y * 256 + threadIdx.x) >> a.lg_lanes), what = 0;
  const int first = (static_cast<int>(threadIdx.x) & (lanes - 1)) * W;
  if (head >= a.q_heads + 2 * a.d.Hk) return;
  if (head >= a.q_heads) {
    head -= a.q_heads;
    what = 1;
    if (head >= a.d.Hk) {
      head -= a.d.Hk;
      what = 2;
    }
  }
  const bool piece = first < a.d.D;  // (the others only take part in the sum)
  const int64_t stride = a.stride[what];
  const E *const src = static_cast<const E *>(a.src[what]) + first_token * stride + static_cast<int64_t>(head) * a.d.D;
  E *const out = what == 0 ? static_cast<E *>(a.q_out) + (static_cast<int64_t>(first_token) * a.d.H + head) * a.d.D + first
                           : static_cast<E *>(a.cache[what - 1]) + (static_cast<int64_t>(head) << a.d.lg_page) * a.d.D + first;
  const int64_t out_stride = static_cast<int64_t>(a.d.H) * a.d.D;
  const int half = a.rope.half;
  const bool rotated = what < 2 && first < 2 * half && piece, second = !a.rope.interleaved && first >= half;
  const bool split = kWhole && rotated && !a.rope.interleaved;  // pairs with another piece
  const int partner = second ? first - half : first + half, pair = a.rope.interleaved ? first / 2 : second ? first - half : first;
  const float *const weight = a.weight[what == 0 ? 0 : 1];
  float w[W], wp[W];
#pragma unroll
  for (int i = 0; i < W; ++i) w[i] = wp[i] = 0.f;
  if (what < 2 && piece) {
    load_rope<W>(weight + first, w);
    if (split) load_rope<W>(weight + partner, wp);
  }
  u32x4 q[kMostTokens], other[kMostTokens];
  Place at[kMostTokens];
#pragma unroll
  for (int k = 0; k < kMostTokens; ++k) {
    at[k].pos = -1;
    q[k] = other[k] = u32x4{0u, 0u, 0u, 0u};
    if (k >= tokens) continue;
    at[k] = place[k];
    if (at[k].pos < 0 || (what > 0 && at[k].slot < 0)) {
      at[k].pos = -1;
      continue;
    }
    const E *const row = src + k * stride;
    if (piece) q[k] = *reinterpret_cast<const u32x4 *>(row + first);
    if (split) other[k] = *reinterpret_cast<const u32x4 *>(row + partner);
  }
#pragma unroll
  for (int k = 0; k < kMostTokens; ++k) {
    if (at[k].pos < 0) continue;  // (alike for the lanes of a head)
    if (what < 2) {
      float v[W], r[W];
      unpack<kBf16>(q[k], v);
      float sum = 0.f;
#pragma unroll
      for (int i = 0; i < W; ++i) sum = fmaf(v[i], v[i], sum);
      for (int m = 1; m < lanes; m <<= 1) sum += __shfl_xor(sum, m);
      const float scale = 1.f / sqrtf(fmaf(sum, a.inv_headdim, a.eps));
#pragma unroll
      for (int i = 0; i < W; ++i) r[i] = v[i] = v[i] * scale * w[i];
      if (rotated) {
        const float *const cs = a.rope.cos + static_cast<int64_t>(at[k].pos) * half, *const sn = a.rope.sin + static_cast<int64_t>(at[k].pos) * half;
        if (split) {
          float o[W], c[W], s[W];
          unpack<kBf16>(other[k], o);
          load_rope<W>(cs + pair, c);
          load_rope<W>(sn + pair, s);
#pragma unroll
          for (int i = 0; i < W; ++i) {
            const float u = o[i] * scale * wp[i];
            r[i] = fmaf(v[i], c[i], second ? u * s[i] : -u * s[i]);
          }
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
          const E *const row = src + k * stride;
#pragma unroll
          for (int i = 0; i < W; ++i) {
            const int c = first + i;
            if (c < 2 * half) {
              const bool b = a.rope.interleaved ? (c & 1) : c >= half;  // the second of its pair
              const int p = a.rope.interleaved ? c >> 1 : b ? c - half : c;
              const int mate = a.rope.interleaved ? c ^ 1 : b ? c - half : c + half;
              const float u = value(row[mate]) * scale * weight[mate];
              r[i] = fmaf(v[i], cs[p], b ? u * sn[p] : -u * sn[p]);
            }
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
    if (piece) *reinterpret_cast<u32x4 *>(out + (what == 0 ? k * out_stride : at[k].slot * a.d.D)) = q[k];
  }
}

int lg_lanes_of(const AttnDims &d) {
  const int pieces = d.D / (d.bf16 ? 8 : 4);
  int lg = 0;
  while ((1 << lg) < pieces) ++lg;
  return lg;
}
int64_t parts_of(const AttnDims &d, bool queries) {
  return (((queries ? d.H : 0) + int64_t{2} * d.Hk) * (int64_t{1} << lg_lanes_of(d)) + 255) / 256;
}
int run_of(const AttnDims &d, int64_t parts) {
  return static_cast<int>(std::max<int64_t>(1, std::min<int64_t>(kMostTokens, d.T * parts / kFewWorkgroups)));
}

}  // namespace

bool attn_append_norm_fits(const AttnDims &d, bool queries) {
  const int64_t parts = parts_of(d, queries);
  const int run = run_of(d, parts);
  return parts <= 65535 && (d.T + int64_t{run} - 1) / run * parts <= kMostWorkgroups256;
}

hipError_t launch_attn_append_norm(const AttnDims &d, const Rope &rope, const int32_t *cu, const int32_t *lens, const int32_t *table,
                                   const void *q, int64_t q_stride, const void *k, int64_t k_stride, const void *v, int64_t v_stride,
                                   const float *q_weight, const float *k_weight, float eps, void *q_out, void *k_cache, void *v_cache,
                                   hipStream_t stream) {
  AppendNormArgs a = {};
  a.src[0] = q;
  a.src[1] = k;
  a.src[2] = v;
  a.stride[0] = q_stride;
  a.stride[1] = k_stride;
  a.stride[2] = v_stride;
  a.weight[0] = q_weight;
  a.weight[1] = k_weight;
  a.q_out = q_out;
  a.cache[0] = k_cache;
  a.cache[1] = v_cache;
  a.cu = cu;
  a.lens = lens;
  a.table = table;
  a.d = d;
  a.rope = rope;
  a.eps = eps;
  a.inv_headdim = 1.f / static_cast<float>(d.D);
  a.lg_lanes = lg_lanes_of(d);
  a.q_heads = q != nullptr ? d.H : 0;
  const int64_t parts = parts_of(d, q != nullptr);
  a.run = run_of(d, parts);
  const dim3 grid((d.T + a.run - 1) / a.run, static_cast<unsigned>(parts));
  const int width = rope.interleaved ? 2 * rope.half : rope.half;
  const bool whole = width % (d.bf16 ? 8 : 4) == 0;
  if (d.bf16 && whole)
    hipLaunchKernelGGL((append_norm_kernel<true, true>), grid, dim3(256), 0, stream, a);
  else if (d.bf16)
    hipLaunchKernelGGL((append_norm_kernel<true, false>), grid, dim3(256), 0, stream, a);
  else if (whole)
    hipLaunchKernelGGL((append_norm_kernel<false, true>), grid, dim3(256), 0, stream, a);
  else
    hipLaunchKernelGGL((append_norm_kernel<false, false>), grid, dim3(256), 0, stream, a);
  return hipGetLastError();
}

}  // namespace ssd
