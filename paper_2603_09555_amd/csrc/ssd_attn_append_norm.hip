// Appends new tokens' keys and values to a paged cache; heads of queries and keys are normalised and rotated by their positions
// on the way:
//
//   u = v rsqrt(mean(v^2) + eps) weight        over the headdim values of a head
//   pair (a, c) of u:  (a cos - c sin, c cos + a sin),  cos, sin = rope[p][pair],  p = seq_lens[b] - (new tokens of b) + j
//   key, value  ->  page table[b][p / page_size], slot p % page_size;  rounded once
//
// A copy in effect, like the append without norms.  A head is held by as many neighbouring lanes as it has pieces of 16 bytes
// (rounded up to a power of two), so that the sum of its squares stays within a wave.  A wave takes some heads of one token, all of
// them queries, or keys, or values, 64 pieces at a time: what a lane needs beside its piece -- its weights, and the cosines and sines
// of its pairs, which are four times the piece -- is the same for all its heads and asked for once.  A piece that holds one half of its
// pairs brings the other halves' piece with it, which a lane nearby brings too, from the first-level cache.
//
// 12 prompts, 16310 tokens, 40 heads over 8 of 64, bf16: 56 us, 4.2 TB/s (87 where each piece asked for its own cosines, sines and
// weights), fp32: 94; 64 single tokens, 32 heads over 8 of 128: 4.4 us; 1023 tokens in fp32 5.1.  Heads of 80, bf16: 85 us with 32 or 80
// values rotated, 292 with 40: rotated halves whose pieces hold values of both are joined value by value, four loads each.
#include <algorithm>

#include "ssd_attn_append.hpp"

namespace ssd {
namespace {

constexpr int kBatch = 2;          // heads whose pieces a lane has on their way at a time
constexpr int kMostTurns = 8;      // heads a lane
constexpr int64_t kWaves = 4096;  // from twice as many on lanes take several heads

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
  int turns;               // heads a lane, at most
  int units[2], all_units; // waves that a token's queries take (none: 0), its keys or its values; all of them
  uint32_t inv_all_units;
};

// The sum over the 2^lg neighbouring lanes of a head, in all of them.  Within a row of 16 without LDS: neighbours, pairs, halves
// and rows mirrored, in each of which every group of lanes has its sum already.
template <int kControl>
__device__ __forceinline__ float moved(float v) {
  return __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(v), kControl, 0xf, 0xf, false));
}
__device__ __forceinline__ float sum_of_head(float v, int lg) {
  if (lg > 0) v += moved<0xb1>(v);   // lanes 1 0 3 2
  if (lg > 1) v += moved<0x4e>(v);   // lanes 2 3 0 1
  if (lg > 2) v += moved<0x141>(v);  // 7 .. 0
  if (lg > 3) v += moved<0x140>(v);  // 15 .. 0
  if (lg > 4) v += __shfl_xor(v, 16);
  if (lg > 5) v += __shfl_xor(v, 32);
  return v;
}

// kWhole: pieces lie in one half of the pairs (interleaved pairs: in the rotated part) or outside it.
template <bool kBf16, bool kWhole>
__global__ __launch_bounds__(256) void append_norm_kernel(const AppendNormArgs a) {
  using E = Element<kBf16>;
  constexpr int W = 16 / sizeof(E);
  // this wave's token, and which heads of what
  const int lane = threadIdx.x & 63, wave = blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
  const int token = quotient(wave, a.all_units, a.inv_all_units);
  if (token >= a.d.T) return;
  int unit = wave - token * a.all_units, what = 0;
  if (unit >= a.units[0]) {
    unit -= a.units[0];
    what = 1;
    if (unit >= a.units[1]) {
      unit -= a.units[1];
      what = 2;
    }
  }
  const Token t = find_token(a.d, a.cu, a.lens, token);
  if (t.pos < 0) return;
  const int64_t slot = what == 0 ? 0 : slot_of(a.d, a.table, t.seq, t.pos, 0);  // cache row of key head 0
  if (slot < 0) return;
  const int heads = what == 0 ? a.d.H : a.d.Hk, at_once = 64 >> a.lg_lanes;
  const int first_head = unit * a.turns * at_once + (lane >> a.lg_lanes), first = (lane & ((1 << a.lg_lanes) - 1)) * W;
  const bool piece = first < a.d.D;  // (the others only take part in the sum)
  const E *const src = static_cast<const E *>(a.src[what]) + token * a.stride[what];
  E *const out = what == 0 ? static_cast<E *>(a.q_out) + static_cast<int64_t>(token) * a.d.H * a.d.D : static_cast<E *>(a.cache[what - 1]) + slot * a.d.D;
  const int64_t out_stride = what == 0 ? a.d.D : static_cast<int64_t>(a.d.D) << a.d.lg_page;  // between heads
  const int half = a.rope.half;
  const bool rotated = what < 2 && first < 2 * half && piece, second = !a.rope.interleaved && first >= half;
  const bool split = kWhole && rotated && !a.rope.interleaved;  // pairs with another piece
  const int partner = second ? first - half : first + half, pair = a.rope.interleaved ? first / 2 : second ? first - half : first;
  const int64_t angles = static_cast<int64_t>(t.pos) * half;
  const float *const weight = a.weight[what == 0 ? 0 : 1];
  // weights, cosines, and sines as they join: the other one's weight with them, and their sign
  float w[W], cs[W], sn[W];
#pragma unroll
  for (int i = 0; i < W; ++i) w[i] = cs[i] = sn[i] = 0.f;
  if (what < 2 && piece) {
    load_rope<W>(weight + first, w);
    if (split) {
      float wp[W];
      load_rope<W>(weight + partner, wp);
      load_rope<W>(a.rope.cos + angles + pair, cs);
      load_rope<W>(a.rope.sin + angles + pair, sn);
#pragma unroll
      for (int i = 0; i < W; ++i) sn[i] = second ? sn[i] * wp[i] : -sn[i] * wp[i];
    } else if (kWhole && rotated) {
      load_rope<W / 2>(a.rope.cos + angles + pair, cs);
      load_rope<W / 2>(a.rope.sin + angles + pair, sn);
    }
  }
  for (int turn = 0; turn < a.turns; turn += kBatch) {
    u32x4 q[kBatch], other[kBatch];
    int head[kBatch];
#pragma unroll
    for (int k = 0; k < kBatch; ++k) {
      head[k] = turn + k < a.turns ? first_head + (turn + k) * at_once : heads;
      q[k] = other[k] = u32x4{0u, 0u, 0u, 0u};
      if (head[k] >= heads || !piece) continue;
      const E *const row = src + static_cast<int64_t>(head[k]) * a.d.D;
      q[k] = *reinterpret_cast<const u32x4 *>(row + first);
      if (split) other[k] = *reinterpret_cast<const u32x4 *>(row + partner);
    }
#pragma unroll
    for (int k = 0; k < kBatch; ++k) {
      if (head[k] >= heads) continue;  // (alike for the lanes of a head)
      if (what < 2) {
        float v[W], r[W];
        unpack<kBf16>(q[k], v);
        float sum = 0.f;
#pragma unroll
        for (int i = 0; i < W; ++i) sum = fmaf(v[i], v[i], sum);
        const float scale = __builtin_amdgcn_rsqf(fmaf(sum_of_head(sum, a.lg_lanes), a.inv_headdim, a.eps));
#pragma unroll
        for (int i = 0; i < W; ++i) r[i] = v[i] = v[i] * scale * w[i];
        if (split) {
          float o[W];
          unpack<kBf16>(other[k], o);
#pragma unroll
          for (int i = 0; i < W; ++i) r[i] = fmaf(v[i], cs[i], o[i] * scale * sn[i]);
        } else if (kWhole && rotated) {
#pragma unroll
          for (int i = 0; i < W; i += 2) {
            r[i] = fmaf(v[i], cs[i / 2], -v[i + 1] * sn[i / 2]);
            r[i + 1] = fmaf(v[i + 1], cs[i / 2], v[i] * sn[i / 2]);
          }
        } else if (rotated) {
          const E *const row = src + static_cast<int64_t>(head[k]) * a.d.D;
#pragma unroll
          for (int i = 0; i < W; ++i) {
            const int e = first + i;
            if (e < 2 * half) {
              const bool b = a.rope.interleaved ? (e & 1) : e >= half;  // the second of its pair
              const int p = a.rope.interleaved ? e >> 1 : b ? e - half : e;
              const int mate = a.rope.interleaved ? e ^ 1 : b ? e - half : e + half;
              const float u = value(row[mate]) * scale * weight[mate], sine = a.rope.sin[angles + p];
              r[i] = fmaf(v[i], a.rope.cos[angles + p], b ? u * sine : -u * sine);
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
      if (piece) *reinterpret_cast<u32x4 *>(out + head[k] * out_stride + first) = q[k];
    }
  }
}

int lg_lanes_of(const AttnDims &d) {
  const int pieces = d.D / (d.bf16 ? 8 : 4);
  int lg = 0;
  while ((1 << lg) < pieces) ++lg;
  return lg;
}
// Waves a token, by its queries and its keys (or values).
struct Units {
  int turns, queries, keys;
  int64_t all() const { return queries + int64_t{2} * keys; }
};
Units units_of(const AttnDims &d, bool queries) {
  const int at_once = 64 >> lg_lanes_of(d);
  const auto units = [&](int heads, int turns) { return (heads + at_once * turns - 1) / (at_once * turns); };
  const int64_t waves = d.T * (units(queries ? d.H : 0, 1) + int64_t{2} * units(d.Hk, 1));
  Units u = {};
  u.turns = static_cast<int>(std::max<int64_t>(1, std::min<int64_t>(kMostTurns, waves / kWaves)));
  u.queries = units(queries ? d.H : 0, u.turns);
  u.keys = units(d.Hk, u.turns);
  return u;
}

}  // namespace

bool attn_append_norm_fits(const AttnDims &d, bool queries) { return (d.T * units_of(d, queries).all() + 3) / 4 <= kMostWorkgroups256; }

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
  const Units u = units_of(d, q != nullptr);
  a.turns = u.turns;
  a.units[0] = u.queries;
  a.units[1] = u.keys;
  a.all_units = static_cast<int>(u.all());
  a.inv_all_units = inverse_of(a.all_units);
  const dim3 grid(static_cast<unsigned>((d.T * u.all() + 3) / 4));
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
