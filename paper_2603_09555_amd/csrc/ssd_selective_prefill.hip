// Selective state space scan of a packed batch of prompts.  For every channel c and state n of a sequence, token by token:
//
//   d = step(dt[t][c]),  h[c][n] = exp(d A[c][n]) h[c][n] + d x[t][c] B[t][n]
//   y[t][c] = (sum_n C[t][n] h[c][n] + D[c] x[t][c]) silu(z[t][c])
//
// The decay differs from state to state, so nothing here is a matrix product.  Bound by the vector unit: an exponential, two issue
// slots on this card (16 of them 154 cycles a wave, 16 fused products 73), and four products for each token, channel and state, where
// a matrix instruction for d x B would save a tenth (it does not overlap with them).
//
// Two kernels: a lane is a channel and holds states of it in registers, or a lane is a state (see by_state_kernel).  There are too few
// channels to fill the chip either way, so time is cut into segments of the packed tokens, whatever sequences these belong to:
//
//   states:  the state at each segment's end, from zero, or from h0 where the last sequence in it begins there, and the sum of
//            that stretch's step sizes (the decay across it is exp(A sum))
//   carry:   the state that enters each segment, one chain a channel and state
//   scan:    the outputs, from the state that enters
//
// A segment whose last token ends a sequence (or is in none) needs no states pass, so that batches of short prompts do little
// twice.  Where all tokens are one segment only the scan runs.  States, sums and step sizes are fp32; y is rounded once.
//
// 16 states, bf16: 16384 tokens x 5120 channels 542 us (322 million issue slots of both passes are 525 at 2.4 GHz; under a profiler
// states 244, carry 15, scan 344), 9938 tokens of 12 prompts 340, 61 tokens x 1536 channels 5.7.  States updated in place: the same.
// fp32, 16384 x 5120: 656; 360 million slots, 585 us: the compiler copies B and C, read for the next token, into vector registers, one or
// two moves a state.  fp32, 2048 x 1536: 46, of which the slots, 17 million, are 28; three launches and trips to memory that some four
// waves a SIMD do not hide are the rest.
#include <algorithm>
#include <type_traits>
#include <utility>

#include "ssd_selective.hpp"

namespace ssd {
namespace {

// B and C as the kernels read them: a row's states are aligned to 4 bytes and as many as the waves hold.
struct Rows {
  const void *b, *c;
  int64_t b_stride, c_stride;  // in elements
};

constexpr float kNothing = -__builtin_inff();

struct ScanArgs {
  SelectiveArgs a;
  Rows rows;
  const int32_t *cu;
  const float *h0;
  float *final_state;
  float *entering;   // (segments, N, C): at a segment's end (states), then the state that enters the next one (carry)
  float *steps;      // (segments, C): sum of the step sizes; kNothing: the state at the end owes nothing to the segments before
  float *begun;      // (segments, N, C): h0 of the sequence that begins in the segment and outlasts it; null: read h0
  SelectiveDims d;
  int segment;       // tokens
  int segments;
};

// The last sequence that begins in front of a token (-1: none).
__device__ __forceinline__ int last_before(const int32_t *cu, int B, int token) {
  int last = -1, behind = B;
  while (behind - last > 1) {
    const int q = (last + behind) / 2;
    if (cu[q] < token) last = q;
    else behind = q;
  }
  return last;
}

// A stride that the compiler cannot multiply in advance: eight rows of every tensor ahead, in registers that it then lacks.
__device__ __forceinline__ uint32_t stride_of(uint32_t v) {
  asm volatile("" : "+s"(v));
  return v;
}

// Values of a row that all lanes of a wave read alike, through the scalar cache.
template <bool kBf16, int NS>
struct Uniform {
  static constexpr int kWords = kBf16 ? NS / 2 : NS;
  uint32_t w[kWords];
  __device__ __forceinline__ void load(const void *row) {
    typedef const __attribute__((address_space(4))) uint32_t *Words;
    const Words p = (Words)(uintptr_t)row;
#pragma unroll
    for (int i = 0; i < kWords; ++i) w[i] = p[i];
  }
  __device__ __forceinline__ float of(int n) const {
    if (!kBf16) return __uint_as_float(w[n % kWords]);
    return __uint_as_float(n % 2 ? w[(n / 2) % kWords] & 0xffff0000u : w[(n / 2) % kWords] << 16);
  }
};

typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef __amdgpu_buffer_rsrc_t Rsrc;
__device__ __forceinline__ Rsrc buffer_at(const void *base) {
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<void *>(base), 0, 0x7fffffff, 0x00020000);
}
constexpr uint32_t kNowhere = 0x80000000u;  // an offset that no such buffer has: a store there is dropped

// A value of either type, as it is in memory until it is used.
template <bool kBf16>
__device__ __forceinline__ uint32_t load_raw(Rsrc r, uint32_t lane_at, uint32_t row_at) {
  if constexpr (kBf16) return static_cast<uint16_t>(__builtin_amdgcn_raw_buffer_load_b16(r, lane_at, row_at, 0));
  else return __builtin_amdgcn_raw_buffer_load_b32(r, lane_at, row_at, 0);
}
template <bool kBf16>
__device__ __forceinline__ float to_float(uint32_t raw) {
  return __uint_as_float(kBf16 ? raw << 16 : raw);
}
__device__ __forceinline__ float value(float v) { return v; }
__device__ __forceinline__ float value(uint16_t v) { return bf16_bits_to_f32(v); }
__device__ __forceinline__ void put(float *p, float v) { *p = v; }
__device__ __forceinline__ void put(uint16_t *p, float v) { *p = __builtin_bit_cast(uint16_t, static_cast<__bf16>(v)); }
template <bool kBf16>
__device__ __forceinline__ void store(Rsrc r, uint32_t lane_at, uint32_t row_at, float v) {
  if constexpr (kBf16) __builtin_amdgcn_raw_buffer_store_b16(__builtin_bit_cast(uint16_t, static_cast<__bf16>(v)), r, lane_at, row_at, 0);
  else __builtin_amdgcn_raw_buffer_store_b32(__float_as_uint(v), r, lane_at, row_at, 0);
}

// What either kernel does with a segment s, of tokens [t0, t1).  A sequence has `size` states; this lane's channel begins at slot in the
// workspace's arrays and at `at` in a sequence's states: `load` and `save` are told which of the two an address is.
template <bool kStates, typename Load, typename Save, typename Walk, typename Total>
__device__ __forceinline__ void scan_segment(const ScanArgs &a, int s, int t0, int t1, int64_t size, int64_t slot, int64_t at, const Load &load,
                                             const Save &save, const Walk &walk, const Total &total, bool writes_total, int c) {
  const int T = a.d.T;
  int q = kStates || s > 0 ? last_before(a.cu, a.d.B, kStates ? t1 : t0) : 0;
  if constexpr (kStates) {
    int begin = 0, end = 0;
    if (q >= 0) {
      begin = max(a.cu[q], 0);
      end = min(a.cu[q + 1], T);
    }
    const bool goes_on = q >= 0 && begin < t1 && end > t1, begins = begin >= t0;
    load(goes_on && begins && a.h0 ? a.h0 + q * size + at : nullptr, false);
    if (goes_on) {
      if (begins && a.begun) save(a.begun + slot, true);
      walk(max(begin, t0), t1);
    }
    save(a.entering + slot, true);
    const float sum = total();
    if (writes_total) a.steps[static_cast<int64_t>(s) * a.d.C + c] = goes_on && !begins ? sum : kNothing;
  } else {
    // the sequence that goes on into this segment, if any, and those that begin in it (at its end, too, if it is the last)
    const int last = s == a.segments - 1 ? T : t1 - 1;
    q = max(q, 0);
    for (int boundary = a.cu[q], next = a.cu[q + 1]; q < a.d.B; ++q) {
      const int begin = min(max(boundary, 0), T), end = min(next, T);
      if (begin > last) break;
      boundary = next;
      next = a.cu[min(q + 2, a.d.B)];  // (on its way while this sequence is walked)
      const bool begins = begin >= t0, kept = begins && end > t1 && a.begun;
      if (!begins && end <= t0) continue;
      load(!begins ? a.entering + slot - size : kept ? a.begun + slot : a.h0 ? a.h0 + q * size + at : nullptr, !begins || kept);
      walk(max(begin, t0), min(end, t1));
      if (end <= t1) save(a.final_state + q * size + at, false);
    }
  }
}

constexpr int block_of(int waves) { return waves >= 4 ? 16 : 8; }
constexpr int waves_a_simd(int states) { return states <= 16 ? 4 : 2; }

// kIo, kDt, kBc: bf16 (x, z, y; dt; rows of B and C).  NS states a wave, W waves for a channel's states.  kStates: the states
// pass.
//
// Tokens are taken in blocks of eight or sixteen.  B and C are the same for all of a wave's lanes and come through the scalar unit.
// A wave turns the rows of its share of a block's tokens into step sizes and inflows, which go to all waves through LDS, and into skip
// terms and gates, which it keeps; then it asks for its rows of the next block.  The waves walk the block's tokens one by one, each on
// its states, with the next token's step, inflow, B and C on their way, and leave the parts of the outputs' sums in LDS, which the wave
// that prepared a token adds up.
template <bool kIo, bool kDt, bool kBc, int NS, int W, bool kStates>
__global__ __launch_bounds__(64 * W, kStates ? 1 : waves_a_simd(NS)) void by_channel_kernel(const ScanArgs a) {
  constexpr int kBlock = block_of(W), kOwn = kBlock / W;  // tokens of a block; those that a wave prepares and finishes
  static_assert(kBlock % W == 0, "a wave's tokens are as many as any other's");
  constexpr uint32_t kSize = kIo ? 2 : 4, kDtSize = kDt ? 2 : 4, kBcSize = kBc ? 2 : 4;
  __shared__ f32x2 lds_du[kBlock + 1][64];  // (a row more, that is read in advance and not used)
  __shared__ float lds_part[kStates ? 1 : W][kBlock][64];
  const int lane = threadIdx.x & 63, wave = W > 1 ? __builtin_amdgcn_readfirstlane(threadIdx.x / 64) : 0;
  const int n0 = wave * NS;
  const int N = a.d.N, C = a.d.C, T = a.d.T;
  const int c_real = blockIdx.x * 64 + lane, c = min(c_real, C - 1);
  const bool live = c_real < C;
  const int s = blockIdx.y;
  const int t0 = s * a.segment, t1 = min(T, t0 + a.segment);

  // (all loads at once: none behind a branch of its own)
  float A2[NS], h[NS];
#pragma unroll
  for (int n = 0; n < NS; ++n) A2[n] = a.a.A[static_cast<int64_t>(c) * N + min(n0 + n, N - 1)];
#pragma unroll
  for (int n = 0; n < NS; ++n) A2[n] = n0 + n < N ? decay_rate(A2[n]) : 0.f;
  const float bias = a.d.dtx.bias ? a.d.dtx.bias[c] : 0.f, skip = !kStates && a.a.D ? a.a.D[c] : 0.f;
  const bool gated = !kStates && a.a.z != nullptr, softplus_alone = a.d.dtx.softplus && !(a.d.dtx.hi > 0.f);
  float total = 0.f;  // of the step sizes

  auto load_state = [&](const float *from, int stride) {  // states n0.. of this lane's channel, `stride` apart
#pragma unroll
    for (int n = 0; n < NS; ++n) h[n] = 0.f;
    if (from == nullptr) return;
#pragma unroll
    for (int n = 0; n < NS; ++n) h[n] = from[static_cast<int64_t>(min(n0 + n, N - 1)) * stride];
#pragma unroll
    for (int n = 0; n < NS; ++n) h[n] = n0 + n < N ? h[n] : 0.f;
  };
  auto store_state = [&](float *to, int stride) {
#pragma unroll
    for (int n = 0; n < NS; ++n)
      if (n0 + n < N && live) to[static_cast<int64_t>(n0 + n) * stride] = h[n];
  };

  // tokens [from, to), which are of one sequence
  auto walk = [&](int from, int to) __attribute__((always_inline)) {
    if (from >= to) return;
    uint32_t raw_x[kOwn], raw_dt[kOwn], raw_z[kOwn];
    auto request = [&](int tb) __attribute__((always_inline)) {
      const Rsrc rx = buffer_at(static_cast<const char *>(a.a.x) + static_cast<int64_t>(tb) * C * kSize);
      const Rsrc rdt = buffer_at(static_cast<const char *>(a.a.dt) + static_cast<int64_t>(tb) * C * kDtSize);
      const uint32_t stride = stride_of(C);
#pragma unroll
      for (int i = 0; i < kOwn; ++i) {
        const uint32_t at = min(wave * kOwn + i, to - 1 - tb) * stride;  // (surplus ones: the last row)
        raw_x[i] = load_raw<kIo>(rx, c * kSize, at * kSize);
        raw_dt[i] = load_raw<kDt>(rdt, c * kDtSize, at * kDtSize);
      }
      if (gated) {
        const Rsrc rz = buffer_at(static_cast<const char *>(a.a.z) + tb * a.a.z_stride * kSize);
        const uint32_t stride = stride_of(static_cast<uint32_t>(a.a.z_stride) * kSize);
#pragma unroll
        for (int i = 0; i < kOwn; ++i) raw_z[i] = load_raw<kIo>(rz, c * kSize, min(wave * kOwn + i, to - 1 - tb) * stride);
      }
    };
    const uint32_t b_step = static_cast<uint32_t>(a.rows.b_stride) * kBcSize, c_step = static_cast<uint32_t>(a.rows.c_stride) * kBcSize;
    const char *b_row = static_cast<const char *>(a.rows.b) + (from * a.rows.b_stride + n0) * kBcSize;
    const char *c_row = static_cast<const char *>(a.rows.c) + (from * a.rows.c_stride + n0) * kBcSize;
    int rows_left = to - from;  // from b_row, c_row on
    Uniform<kBc, NS> b_next, c_next;
    auto request_row = [&]() __attribute__((always_inline)) {  // (surplus ones: the last row)
      b_next.load(b_row);
      if constexpr (!kStates) c_next.load(c_row);
      if (--rows_left > 0) {
        b_row += b_step;
        c_row += c_step;
      }
    };
    request_row();
    request(from);
    for (int tb = from; tb < to; tb += kBlock) {
      const int count = min(kBlock, to - tb);
      float d_own[kOwn], sum[kOwn], gate[kOwn];
      if (softplus_alone) {
#pragma unroll
        for (int i = 0; i < kOwn; ++i) d_own[i] = softplus(to_float<kDt>(raw_dt[i]) + bias);
      } else {
#pragma unroll
        for (int i = 0; i < kOwn; ++i) d_own[i] = step_of(to_float<kDt>(raw_dt[i]), bias, a.d.dtx);
      }
#pragma unroll
      for (int i = 0; i < kOwn; ++i) {
        const float x = to_float<kIo>(raw_x[i]);
        lds_du[wave * kOwn + i][lane] = f32x2{d_own[i], d_own[i] * x};
        sum[i] = skip * x;
      }
      if (gated) {
#pragma unroll
        for (int i = 0; i < kOwn; ++i) gate[i] = silu(to_float<kIo>(raw_z[i]));
      }
      if (tb + kBlock < to) request(tb + kBlock);
      if constexpr (W > 1) __syncthreads();
      f32x2 du_next = lds_du[0][lane];
#pragma unroll 2
      for (int i = 0; i < count; ++i) {
        const Uniform<kBc, NS> b_now = b_next, c_now = c_next;
        const float d = du_next[0], u = du_next[1];
        request_row();
        du_next = lds_du[i + 1][lane];
        if constexpr (kStates) total += d;
        float part[2] = {0.f, 0.f};
#pragma unroll
        for (int n = 0; n < NS; ++n) {
          h[n] = fmaf(__builtin_amdgcn_exp2f(d * A2[n]), h[n], u * b_now.of(n));
          if constexpr (!kStates) part[n % 2] = fmaf(c_now.of(n), h[n], part[n % 2]);
        }
        if constexpr (!kStates) lds_part[wave][i][lane] = part[0] + part[1];
      }
      if constexpr (W > 1) __syncthreads();
      if constexpr (!kStates) {
        const Rsrc ry = buffer_at(static_cast<char *>(a.a.y) + static_cast<int64_t>(tb) * C * kSize);
        const uint32_t lane_at = live ? c * kSize : kNowhere, stride = stride_of(C * kSize);
#pragma unroll
        for (int i = 0; i < kOwn; ++i)
#pragma unroll
          for (int w = 0; w < W; ++w) sum[i] += lds_part[w][wave * kOwn + i][lane];
        if (gated) {
#pragma unroll
          for (int i = 0; i < kOwn; ++i) sum[i] *= gate[i];
        }
#pragma unroll
        for (int i = 0; i < kOwn; ++i)
          if (wave * kOwn + i < count) store<kIo>(ry, lane_at, (wave * kOwn + i) * stride, sum[i]);
      }
    }
  };

  scan_segment<kStates>(a, s, t0, t1, static_cast<int64_t>(C) * N, static_cast<int64_t>(s) * N * C + c, static_cast<int64_t>(c) * N,
                        [&](const float *from, bool slot) { load_state(from, slot ? C : 1); },
                        [&](float *to, bool slot) { store_state(to, slot ? C : 1); }, walk,
                        [&] { return total; }, wave == 0 && live, c);
}

// The other kernel, for calls of little work: a lane is a state of a channel (S of them, 16 apart), a row of 16 lanes a channel, a wave
// four channels.  That makes sixteen times the waves.  A row's lanes prepare 16 tokens of its channel, one each, and hand step sizes and
// inflows around with the operand's own lane exchange; an output's sum over the states is one over the row's lanes, and 16 tokens' sums
// are made together, each step halving what a lane has, so that a lane ends with its token's.  B and C go through LDS, for the four
// waves of a workgroup: a load for each token and wave would keep the memory pipe busy for longer than the block takes.
template <int kControl>
__device__ __forceinline__ float from_lane(float v) {
  return __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(v), kControl, 0xf, 0xf, true));
}
template <int I>
__device__ __forceinline__ float of_token(float v) {  // lane I's of the row
  return from_lane<0x150 + I>(v);
}
template <int... I, typename F>
__device__ __forceinline__ void each(std::integer_sequence<int, I...>, const F &f) {
  (f(std::integral_constant<int, I>()), ...);
}

template <bool kIo, bool kDt, int S, bool kStates>
__global__ __launch_bounds__(256) void by_state_kernel(const ScanArgs a) {
  constexpr int kBlock = 16;
  __shared__ float lds_rows[2][2][16 * S][kBlock + 4];  // B and C of a block's tokens, of this one and the next
  using E = typename std::conditional<kIo, uint16_t, float>::type;
  using EDt = typename std::conditional<kDt, uint16_t, float>::type;
  const int lane = threadIdx.x & 63, nl = lane & 15;
  const int N = a.d.N, C = a.d.C, T = a.d.T;
  // neighbouring channels, whose rows share cache lines, on one die (workgroups go to the eight of them in turn)
  const int across = gridDim.x, group = across % 8 == 0 ? (blockIdx.x % 8) * (across / 8) + blockIdx.x / 8 : blockIdx.x;
  const int c_real = group * 16 + threadIdx.x / 16, c = min(c_real, C - 1);
  const bool live = c_real < C;
  const int s = blockIdx.y;
  const int t0 = s * a.segment, t1 = min(T, t0 + a.segment);

  float A2[S], h[S];
#pragma unroll
  for (int k = 0; k < S; ++k) A2[k] = a.a.A[static_cast<int64_t>(c) * N + min(16 * k + nl, N - 1)];
#pragma unroll
  for (int k = 0; k < S; ++k) A2[k] = 16 * k + nl < N ? decay_rate(A2[k]) : 0.f;
  const float bias = a.d.dtx.bias ? a.d.dtx.bias[c] : 0.f, skip = !kStates && a.a.D ? a.a.D[c] : 0.f;
  const bool gated = !kStates && a.a.z != nullptr;
  float total = 0.f;  // of the step sizes, this lane's

  auto load_state = [&](const float *from) {  // state 0 of this lane's channel
#pragma unroll
    for (int k = 0; k < S; ++k) h[k] = from ? from[min(16 * k + nl, N - 1)] : 0.f;
#pragma unroll
    for (int k = 0; k < S; ++k) h[k] = 16 * k + nl < N ? h[k] : 0.f;
  };
  auto store_state = [&](float *to) {
#pragma unroll
    for (int k = 0; k < S; ++k)
      if (16 * k + nl < N && live) to[16 * k + nl] = h[k];
  };

  // tokens [from, to), which are of one sequence
  auto walk = [&](int from, int to) __attribute__((always_inline)) {
    if (from >= to) return;
    // the rows of two blocks are on their way: one wave's work on a block takes less than memory does.  Of B and C, which all
    // channels share, a thread brings its states of one token
    E raw_x[2], raw_z[2] = {E(0), E(0)}, raw_b[2][S], raw_c[2][S];
    EDt raw_dt[2];
    const int own_token = threadIdx.x / 16;
    auto request = [&](int tb, int slot) __attribute__((always_inline)) {
      const int64_t t = min(tb + nl, to - 1), r = min(tb + own_token, to - 1);  // (surplus ones: the last row)
      raw_x[slot] = static_cast<const E *>(a.a.x)[t * C + c];
      raw_dt[slot] = static_cast<const EDt *>(a.a.dt)[t * C + c];
      if (gated) raw_z[slot] = static_cast<const E *>(a.a.z)[t * a.a.z_stride + c];
#pragma unroll
      for (int k = 0; k < S; ++k) {
        const int n = min(16 * k + nl, N - 1);
        raw_b[slot][k] = static_cast<const E *>(a.a.B)[r * a.a.b_stride + n];
        if constexpr (!kStates) raw_c[slot][k] = static_cast<const E *>(a.a.C)[r * a.a.c_stride + n];
      }
    };
    // a block of tokens, the first or the second of two
    auto block = [&](int tb, auto which) __attribute__((always_inline)) {
      constexpr int kWhich = decltype(which)::value;
      // this lane's token (behind `to`: a step of nothing)
      const bool there = tb + nl < to;
      const float x = value(raw_x[kWhich]), step = step_of(value(raw_dt[kWhich]), bias, a.d.dtx);
      const float d = there ? step : 0.f, u = there ? step * x : 0.f;
      const float gate = gated ? silu(value(raw_z[kWhich])) : 1.f;
#pragma unroll
      for (int k = 0; k < S; ++k) {
        const bool staged = tb + own_token < to && 16 * k + nl < N;  // (zeros behind `to`: what is there is another sequence's)
        lds_rows[kWhich][0][16 * k + nl][own_token] = staged ? value(raw_b[kWhich][k]) : 0.f;
        if constexpr (!kStates) lds_rows[kWhich][1][16 * k + nl][own_token] = staged ? value(raw_c[kWhich][k]) : 0.f;
      }
      if (tb + 2 * kBlock < to) request(tb + 2 * kBlock, kWhich);
      __syncthreads();
      if constexpr (kStates) total += d;
      float sum[kBlock];
      each(std::make_integer_sequence<int, kBlock / 4>(), [&](auto quarter) {
        constexpr int i0 = decltype(quarter)::value * 4;
        if (i0 > 0 && tb + i0 >= to) {
#pragma unroll
          for (int i = 0; i < 4; ++i) sum[i0 + i] = 0.f;
          return;
        }
        f32x4 b_now[S], c_now[S];
#pragma unroll
        for (int k = 0; k < S; ++k) {
          b_now[k] = *reinterpret_cast<const f32x4 *>(&lds_rows[kWhich][0][16 * k + nl][i0]);
          if constexpr (!kStates) c_now[k] = *reinterpret_cast<const f32x4 *>(&lds_rows[kWhich][1][16 * k + nl][i0]);
        }
        each(std::make_integer_sequence<int, 4>(), [&](auto token) {
          constexpr int i = decltype(token)::value;
          float y = 0.f;
#pragma unroll
          for (int k = 0; k < S; ++k) {
            h[k] = fmaf(__builtin_amdgcn_exp2f(of_token<i0 + i>(d) * A2[k]), h[k], of_token<i0 + i>(u) * b_now[k][i]);
            if constexpr (!kStates) y = fmaf(c_now[k][i], h[k], y);
          }
          sum[i0 + i] = y;
        });
      });
      if constexpr (!kStates) {
        // halves of a row, of eight, of four and of two lanes keep the tokens whose bit they have
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const float low = sum[j] + from_lane<0x140>(sum[j]), high = sum[j + 8] + from_lane<0x140>(sum[j + 8]);
          sum[j] = nl & 8 ? high : low;
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const float low = sum[j] + from_lane<0x141>(sum[j]), high = sum[j + 4] + from_lane<0x141>(sum[j + 4]);
          sum[j] = nl & 4 ? high : low;
        }
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          const float low = sum[j] + from_lane<0x4e>(sum[j]), high = sum[j + 2] + from_lane<0x4e>(sum[j + 2]);
          sum[j] = nl & 2 ? high : low;
        }
        const float low = sum[0] + from_lane<0xb1>(sum[0]), high = sum[1] + from_lane<0xb1>(sum[1]);
        const float y = fmaf(skip, x, nl & 1 ? high : low);
        if (there && live) put(static_cast<E *>(a.a.y) + static_cast<int64_t>(tb + nl) * C + c, gated ? y * gate : y);
      }
    };
    request(from, 0);
    if (from + kBlock < to) request(from + kBlock, 1);
    __syncthreads();  // (the rows of a sequence before)
    for (int tb = from; tb < to; tb += 2 * kBlock) {
      block(tb, std::integral_constant<int, 0>());
      if (tb + kBlock < to) block(tb + kBlock, std::integral_constant<int, 1>());
    }
  };

  scan_segment<kStates>(a, s, t0, t1, static_cast<int64_t>(C) * N, static_cast<int64_t>(s) * C * N + static_cast<int64_t>(c) * N,
                        static_cast<int64_t>(c) * N, [&](const float *from, bool) { load_state(from); },
                        [&](float *to, bool) { store_state(to); }, walk, [&] {
                          float sum = total;
                          sum += from_lane<0xb1>(sum);
                          sum += from_lane<0x4e>(sum);
                          sum += from_lane<0x141>(sum);
                          sum += from_lane<0x140>(sum);
                          return sum;
                        }, nl == 0 && live, c);
}

// The state that enters each segment but the first, in place of the one at the end of the segment before.  Eight segments'
// values are on their way at a time.
__global__ __launch_bounds__(256) void carry_kernel(float *entering, const float *steps, const float *A, int N, int C, int segments, bool by_state) {
  const int64_t i = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x, size = static_cast<int64_t>(N) * C;
  if (i >= size) return;
  const int c = static_cast<int>(by_state ? i / N : i % C), n = static_cast<int>(by_state ? i % N : i / C);
  const float A2 = decay_rate(A[static_cast<int64_t>(c) * N + n]);
  constexpr int kAhead = 8;
  float h = 0.f, sum[kAhead], e[kAhead];
  auto request = [&](int s0) {
#pragma unroll
    for (int k = 0; k < kAhead; ++k) {
      const int s = min(s0 + k, segments - 2);
      sum[k] = steps[static_cast<int64_t>(s) * C + c];
      e[k] = entering[s * size + i];
    }
  };
  request(0);
  for (int s0 = 0; s0 < segments - 1; s0 += kAhead) {
    float out[kAhead];
#pragma unroll
    for (int k = 0; k < kAhead; ++k) out[k] = h = sum[k] == kNothing ? e[k] : fmaf(__builtin_amdgcn_exp2f(sum[k] * A2), h, e[k]);
    if (s0 + kAhead < segments - 1) request(s0 + kAhead);
#pragma unroll
    for (int k = 0; k < kAhead; ++k)
      if (s0 + k < segments - 1) entering[(s0 + k) * size + i] = out[k];
  }
}

// B and C in fp32, states from N up to the waves' zero.
template <typename E>
__global__ __launch_bounds__(256) void rows_kernel(const void *b, const void *c, int64_t b_stride, int64_t c_stride, int N, int padded, int64_t values,
                                                   float *out) {
  const int64_t i = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x;
  if (i >= values) return;
  const int64_t t = i / padded;
  const int n = static_cast<int>(i - t * padded);
  out[i] = n < N ? value(static_cast<const E *>(b)[t * b_stride + n]) : 0.f;
  out[values + i] = n < N ? value(static_cast<const E *>(c)[t * c_stride + n]) : 0.f;
}

// How a call is cut up.
struct Cut {
  bool by_state;
  int states, waves;         // by channel: of a wave, and waves for a channel's; by state: of a lane
  int64_t most_segments;     // that the workspace has room for: never fewer for more tokens
  int segment;               // tokens
  int padded() const { return by_state ? 0 : states * waves; }
};
// `most` segments, of `shortest` tokens or more.
void set_segments(const SelectiveDims &d, int64_t most, int64_t shortest, int block, Cut *c) {
  c->most_segments = std::max<int64_t>(1, most);
  const int64_t least = (d.T + c->most_segments - 1) / c->most_segments;
  const int64_t wanted = std::max<int64_t>(knobs().selective_segment > 0 ? knobs().selective_segment : shortest, least);
  c->segment = static_cast<int>((wanted + block - 1) / block * block);
}
// By channel: eight states a wave (16 cost as much where there is work for them and leave fewer waves where there is not, four cost 20 %
// more), and segments for 16 waves a SIMD, of 48 tokens or more.
Cut cut_by_channel(const SelectiveDims &d) {
  int padded = 8;
  while (padded < d.N) padded *= 2;
  const int64_t groups = (d.C + 63) / 64;
  Cut c = {};
  c.states = std::max(8, padded / 8);
  c.waves = padded / c.states;
  set_segments(d, std::min<int64_t>((d.T + 47) / 48, 16384 / c.waves / groups), 1, block_of(c.waves), &c);
  return c;
}
// By state: segments for four waves a SIMD, of 64 tokens or more, where the two launches in front of the scan cost less than they
// save: 1536 channels, 256 tokens 13.7 us in one segment and 15.7 in four, 512 tokens 24.6 and 19.3 in eight.  To begin a sequence
// takes as long as some 40 tokens, so that a segment shall not hold many: 512 tokens of 32 sequences 68 us in one, 38 in eight.
Cut cut_by_state(const SelectiveDims &d) {
  Cut c = {};
  c.by_state = true;
  c.states = d.N <= 16 ? 1 : d.N <= 32 ? 2 : 4;
  const int64_t waves = (d.C + 3) / 4;
  const bool one = d.T + int64_t{40} * (d.B - 1) <= 384 + waves / 4;
  const int64_t shortest = one ? d.T : std::min<int64_t>(64, int64_t{4} * d.T / d.B);
  set_segments(d, std::min<int64_t>((d.T + 15) / 16, 4096 / waves), shortest, 16, &c);
  return c;
}
// A lane a state up to 2^26 states of all tokens: 16 states, us by state and by channel, 1536 channels, 61 tokens 5.6 / 21, 512 19 / 35,
// 2048 (fp32) 46 / 52; 5120 channels, 512 tokens 36 / 43, 2048 116 / 103.  At 2^26, bf16: 16 states, 256 to 8192 channels 60 / 87, 61 / 70,
// 63 / 64, 62 / 63, 37 / 53; 32 states 49 / 52, 64 states 40 / 56.  At 2^27 by state takes 0.88 to 1.3 of by channel.  8 states leave half
// of a row's lanes without one: 1536 channels, 2730 tokens (2^25) 62 / 54, 5461 tokens (2^26) 111 / 70.
constexpr int kMostByState = 64;  // states of a channel
Cut cut_of(const SelectiveDims &d) {
  const int64_t work = static_cast<int64_t>(d.T) * d.C * d.N;
  const int knob = knobs().selective_by_state;
  return d.N <= kMostByState && (knob == 1 || (knob == 0 && work < (1 << 26))) ? cut_by_state(d) : cut_by_channel(d);
}
int64_t segments_of(const SelectiveDims &d, const Cut &c) { return (static_cast<int64_t>(d.T) + c.segment - 1) / c.segment; }

// Parts of the workspace, in bytes.
struct Plan {
  size_t rows, entering, steps, begun, total;
};
Plan plan_of(const SelectiveDims &d, const Cut &c) {
  Plan p = {};
  const size_t segments = static_cast<size_t>(c.most_segments);
  size_t at = 0;
  const auto take = [&](size_t bytes) {
    const size_t was = at;
    at += round_up(bytes, 256);
    return was;
  };
  p.rows = take(static_cast<size_t>(d.T) * 2 * c.padded() * 4);
  p.entering = take(segments > 1 ? segments * d.N * d.C * 4 : 0);
  p.steps = take(segments > 1 ? segments * d.C * 4 : 0);
  p.begun = take(segments > 1 ? segments * d.N * d.C * 4 : 0);
  p.total = at;
  return p;
}

// The launches of a call by states and scan kernels of either kind.
template <typename States, typename Scan>
hipError_t launch_passes(const ScanArgs &a, bool by_state, const States &states, const Scan &scan, hipStream_t stream) {
  if (a.segments > 1) {
    states();
    if (const hipError_t e = hipGetLastError(); e != hipSuccess) return e;
    const dim3 grid(static_cast<unsigned>((static_cast<int64_t>(a.d.C) * a.d.N + 255) / 256));
    hipLaunchKernelGGL(carry_kernel, grid, dim3(256), 0, stream, a.entering, a.steps, a.a.A, a.d.N, a.d.C, a.segments, by_state);
    if (const hipError_t e = hipGetLastError(); e != hipSuccess) return e;
  }
  scan();
  return hipGetLastError();
}

template <bool kIo, bool kDt, int S>
hipError_t launch_by_state(const ScanArgs &a, hipStream_t stream) {
  const unsigned groups = (a.d.C + 15) / 16;
  return launch_passes(
      a, true, [&] { hipLaunchKernelGGL((by_state_kernel<kIo, kDt, S, true>), dim3(groups, a.segments - 1), dim3(256), 0, stream, a); },
      [&] { hipLaunchKernelGGL((by_state_kernel<kIo, kDt, S, false>), dim3(groups, a.segments), dim3(256), 0, stream, a); }, stream);
}
template <bool kIo, bool kDt>
hipError_t launch_by_state(const ScanArgs &a, const Cut &c, hipStream_t stream) {
  if (c.states == 1) return launch_by_state<kIo, kDt, 1>(a, stream);
  if (c.states == 2) return launch_by_state<kIo, kDt, 2>(a, stream);
  return launch_by_state<kIo, kDt, 4>(a, stream);
}

template <bool kIo, bool kDt, bool kBc, int NS, int W>
hipError_t launch_split(const ScanArgs &a, hipStream_t stream) {
  const unsigned groups = (a.d.C + 63) / 64;
  return launch_passes(
      a, false, [&] { hipLaunchKernelGGL((by_channel_kernel<kIo, kDt, kBc, NS, W, true>), dim3(groups, a.segments - 1), dim3(64 * W), 0, stream, a); },
      [&] { hipLaunchKernelGGL((by_channel_kernel<kIo, kDt, kBc, NS, W, false>), dim3(groups, a.segments), dim3(64 * W), 0, stream, a); }, stream);
}
template <bool kIo, bool kDt, bool kBc>
hipError_t launch_by_channel(const ScanArgs &a, const Cut &c, hipStream_t stream) {
  if (c.waves == 1) return launch_split<kIo, kDt, kBc, 8, 1>(a, stream);
  if (c.waves == 2) return launch_split<kIo, kDt, kBc, 8, 2>(a, stream);
  if (c.waves == 4) return launch_split<kIo, kDt, kBc, 8, 4>(a, stream);
  if (c.states == 8) return launch_split<kIo, kDt, kBc, 8, 8>(a, stream);
  if (c.states == 16) return launch_split<kIo, kDt, kBc, 16, 8>(a, stream);
  return launch_split<kIo, kDt, kBc, 32, 8>(a, stream);
}

}  // namespace

// Whether no launch of a call has 2^32 threads or more.
bool selective_prefill_fits(const SelectiveDims &d) {
  const Cut c = cut_by_channel(d), e = cut_by_state(d);
  const int64_t groups = (d.C + 63) / 64, limit = int64_t{1} << 32;
  return c.most_segments <= 65535 && groups * c.most_segments * c.waves * 64 < limit && (static_cast<int64_t>(d.T) + 256) * c.padded() < limit &&
         (d.N > kMostByState || (e.most_segments <= 65535 && groups * e.most_segments * 1024 < limit));
}

// (of either kind: the choice between them is none of the caller's)
size_t selective_prefill_workspace_bytes(const SelectiveDims &d) {
  const size_t one = plan_of(d, cut_by_channel(d)).total;
  return d.N > kMostByState ? one : std::max(one, plan_of(d, cut_by_state(d)).total);
}

hipError_t launch_selective_prefill(const SelectiveDims &d, const SelectiveArgs &args, const int32_t *cu, const float *h0, float *final_state,
                                    void *workspace, hipStream_t stream) {
  const Cut s = cut_of(d);
  const Plan p = plan_of(d, s);
  char *const w = static_cast<char *>(workspace);
  ScanArgs a = {};
  a.a = args;
  a.cu = cu;
  a.h0 = h0;
  a.final_state = final_state;
  a.entering = reinterpret_cast<float *>(w + p.entering);
  a.steps = reinterpret_cast<float *>(w + p.steps);
  a.begun = h0 && h0 == final_state ? reinterpret_cast<float *>(w + p.begun) : nullptr;
  a.d = d;
  a.segment = s.segment;
  a.segments = static_cast<int>(segments_of(d, s));
  if (a.segments == 1) a.begun = nullptr;
  if (s.by_state) {
    if (!d.bf16) return launch_by_state<false, false>(a, s, stream);
    return d.dt_bf16 ? launch_by_state<true, true>(a, s, stream) : launch_by_state<true, false>(a, s, stream);
  }
  a.rows = {args.B, args.C, args.b_stride, args.c_stride};
  const bool whole = d.N == s.padded() && ((reinterpret_cast<uintptr_t>(args.B) | reinterpret_cast<uintptr_t>(args.C)) & 3) == 0 &&
                     (!d.bf16 || (args.b_stride % 2 == 0 && args.c_stride % 2 == 0));
  if (!whole) {
    float *const rows = reinterpret_cast<float *>(w + p.rows);
    const int64_t values = static_cast<int64_t>(d.T) * s.padded();
    const dim3 grid(static_cast<unsigned>((values + 255) / 256));
    if (d.bf16)
      hipLaunchKernelGGL((rows_kernel<uint16_t>), grid, dim3(256), 0, stream, args.B, args.C, args.b_stride, args.c_stride, d.N, s.padded(), values, rows);
    else
      hipLaunchKernelGGL((rows_kernel<float>), grid, dim3(256), 0, stream, args.B, args.C, args.b_stride, args.c_stride, d.N, s.padded(), values, rows);
    if (const hipError_t e = hipGetLastError(); e != hipSuccess) return e;
    a.rows = {rows, rows + values, s.padded(), s.padded()};
  }
  if (!d.bf16) return launch_by_channel<false, false, false>(a, s, stream);
  if (d.dt_bf16) return whole ? launch_by_channel<true, true, true>(a, s, stream) : launch_by_channel<true, true, false>(a, s, stream);
  return whole ? launch_by_channel<true, false, true>(a, s, stream) : launch_by_channel<true, false, false>(a, s, stream);
}

}  // namespace ssd
