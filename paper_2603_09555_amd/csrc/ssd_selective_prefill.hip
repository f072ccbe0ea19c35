// Selective state space scan of a packed batch of prompts.  For every channel c and state n of a sequence, token by token:
//
//   d = step(dt[t][c]),  h[c][n] = exp(d A[c][n]) h[c][n] + d x[t][c] B[t][n]
//   y[t][c] = (sum_n C[t][n] h[c][n] + D[c] x[t][c]) silu(z[t][c])
//
// A lane is a channel and holds its states in registers; B and C are the same for all of a wave's lanes and come through the
// scalar unit.
//
// The decay differs from state to state, so nothing here is a matrix product: an exponential (a quarter of the vector rate) and
// four vector operations for each token, channel and state, which bounds the kernel where memory does not.  There are too few
// channels to fill the chip, so time is cut into segments of the packed tokens, whatever sequences these belong to:
//
//   states:  the state at each segment's end, from zero, or from h0 where the last sequence in it begins there, and the sum of
//            that stretch's step sizes (the decay across it is exp(A sum))
//   carry:   the state that enters each segment, one chain a channel and state
//   scan:    the outputs, from the state that enters
//
// A segment whose last token ends a sequence (or is in none) needs no states pass, so that batches of short prompts do little
// twice.  Where all tokens are one segment only the scan runs.
#include <algorithm>
#include <type_traits>

#include "ssd_selective.hpp"

namespace ssd {
namespace {

// B and C as the kernels read them: a row's states are aligned to 4 bytes and as many as the waves hold.
struct Rows {
  const void *b, *c;
  int64_t b_stride, c_stride;  // in elements
};

struct ScanArgs {
  SelectiveArgs a;
  Rows rows;
  const int32_t *cu;
  const float *h0;
  float *final_state;
  float *entering;   // (segments, N, C): at a segment's end (states), then the state that enters the next one (carry)
  float *steps;      // (segments, C): sum of the step sizes; negative: the state at the end owes nothing to the segments before
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
template <bool kBf16>
__device__ __forceinline__ void store(Rsrc r, uint32_t lane_at, uint32_t row_at, float v) {
  if constexpr (kBf16) __builtin_amdgcn_raw_buffer_store_b16(__builtin_bit_cast(uint16_t, static_cast<__bf16>(v)), r, lane_at, row_at, 0);
  else __builtin_amdgcn_raw_buffer_store_b32(__float_as_uint(v), r, lane_at, row_at, 0);
}

constexpr int block_of(int waves) { return waves >= 4 ? 16 : 8; }
constexpr int waves_a_simd(int states) { return states <= 16 ? 4 : 2; }

// kIo, kDt, kBc: bf16 (x, z, y; dt; rows of B and C).  NS states a wave, W waves for a channel's states.  kStates: the states
// pass.
//
// Tokens are taken in blocks of eight.  A wave turns the rows of its share of a block's tokens into step sizes and inflows, which
// go to all waves through LDS, and into skip terms and gates, which it keeps; then it asks for its rows of the next block.  The
// waves walk the block's tokens one by one, each on its states, with the next token's step, inflow, B and C on their way, and
// leave the parts of the outputs' sums in LDS, which the wave that prepared a token adds up.
template <bool kIo, bool kDt, bool kBc, int NS, int W, bool kStates>
__global__ __launch_bounds__(64 * W, kStates ? 1 : waves_a_simd(NS)) void selective_kernel(const ScanArgs a) {
    constexpr int kBlock = block_of(W), kOwn = kBlock / W;  // tokens of a block; those that a wave prepares and finishes
  static_assert(kBlock % W == 0, "a wave's tokens are as many as any other's");
  constexpr uint32_t kSize = kIo ? 2 : 4, kDtSize = kDt ? 2 : 4, kBcSize = kBc ? 2 : 4;
  // Tokens whose B and C are asked for together, while the ones before are worked on: scalar loads come back in any order, so that
  // a wait is for all of them.
  constexpr int kWords = (kStates ? 2 : 4) * Uniform<kBc, NS>::kWords;  // of both sets, a token
  constexpr int kAhead = NS > 4 ? 1 : kWords <= 8 ? 8 : 4, kUnroll = kAhead > 1 ? 1 : 2;
  __shared__ f32x2 lds_du[kBlock + kAhead][64];  // (rows that are read in advance and not used)
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
  for (int n = 0; n < NS; ++n) A2[n] = n0 + n < N ? A2[n] * kLog2e : 0.f;
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
    Uniform<kBc, NS> b_next[kAhead], c_next[kAhead];
    auto request_rows = [&]() __attribute__((always_inline)) {  // (surplus ones: the last row)
#pragma unroll
      for (int k = 0; k < kAhead; ++k) {
        b_next[k].load(b_row);
        if constexpr (!kStates) c_next[k].load(c_row);
        if (--rows_left > 0) {
          b_row += b_step;
          c_row += c_step;
        }
      }
    };
    request_rows();
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
      f32x2 du_next[kAhead];
#pragma unroll
      for (int k = 0; k < kAhead; ++k) du_next[k] = lds_du[k][lane];
#pragma unroll kUnroll
      for (int i0 = 0; i0 < count; i0 += kAhead) {
        Uniform<kBc, NS> b_now[kAhead], c_now[kAhead];
        f32x2 du[kAhead];
#pragma unroll
        for (int k = 0; k < kAhead; ++k) {
          b_now[k] = b_next[k];
          c_now[k] = c_next[k];
          du[k] = du_next[k];
        }
        request_rows();
#pragma unroll
        for (int k = 0; k < kAhead; ++k) du_next[k] = lds_du[i0 + kAhead + k][lane];
#pragma unroll
        for (int k = 0; k < kAhead; ++k) {
          if (k > 0 && i0 + k >= count) break;
          const float d = du[k][0], u = du[k][1];
          if constexpr (kStates) total += d;
          float part[2] = {0.f, 0.f};
#pragma unroll
          for (int n = 0; n < NS; ++n) {
            h[n] = fmaf(__builtin_amdgcn_exp2f(d * A2[n]), h[n], u * b_now[k].of(n));
            if constexpr (!kStates) part[n % 2] = fmaf(c_now[k].of(n), h[n], part[n % 2]);
          }
          if constexpr (!kStates) lds_part[wave][i0 + k][lane] = part[0] + part[1];
        }
      }
      if constexpr (W > 1) __syncthreads();
      if constexpr (!kStates) {
        const Rsrc ry = buffer_at(static_cast<char *>(a.a.y) + static_cast<int64_t>(tb) * C * kSize);
        const uint32_t lane_at = live ? c * kSize : kNowhere, stride = stride_of(C * kSize);
#pragma unroll
        for (int i = 0; i < kOwn; ++i) {
          const int row = wave * kOwn + i;
#pragma unroll
          for (int w = 0; w < W; ++w) sum[i] += lds_part[w][row][lane];
          if (gated) sum[i] *= gate[i];
          if (row < count) store<kIo>(ry, lane_at, row * stride, sum[i]);
        }
      }
    }
  };

  const int64_t slot = (static_cast<int64_t>(s) * N) * C + c;  // of state 0 of this segment and channel
  const int64_t sequence_size = static_cast<int64_t>(C) * N;
  int q = last_before(a.cu, a.d.B, kStates ? t1 : t0);
  if constexpr (kStates) {
    int begin = 0, end = 0;
    if (q >= 0) {
      begin = max(a.cu[q], 0);
      end = min(a.cu[q + 1], T);
    }
    const bool goes_on = q >= 0 && begin < t1 && end > t1, begins = begin >= t0;
    load_state(goes_on && begins && a.h0 ? a.h0 + q * sequence_size + static_cast<int64_t>(c) * N : nullptr, 1);
    if (goes_on) {
      if (begins && a.begun) store_state(a.begun + slot, C);
      walk(max(begin, t0), t1);
    }
    store_state(a.entering + slot, C);
    if (wave == 0 && live) a.steps[static_cast<int64_t>(s) * C + c] = goes_on && !begins ? total : -1.f;
  } else {
    // the sequence that goes on into this segment, if any, and those that begin in it (at its end, too, if it is the last)
    const int last = s == a.segments - 1 ? T : t1 - 1;
    for (q = s == 0 ? 0 : max(q, 0); q < a.d.B; ++q) {
      const int begin = min(max(a.cu[q], 0), T), end = min(a.cu[q + 1], T);
      if (begin > last) break;
      const bool begins = begin >= t0;
      if (!begins && end <= t0) continue;
      if (begins) {
        const bool kept = end > t1 && a.begun;
        load_state(kept ? a.begun + slot : a.h0 ? a.h0 + q * sequence_size + static_cast<int64_t>(c) * N : nullptr, kept ? C : 1);
      } else {
        load_state(a.entering + slot - sequence_size, C);
      }
      walk(max(begin, t0), min(end, t1));
      if (end <= t1) store_state(a.final_state + q * sequence_size + static_cast<int64_t>(c) * N, 1);
    }
  }
}

// The state that enters each segment but the first, in place of the one at the end of the segment before.  Eight segments'
// values are on their way at a time.
__global__ __launch_bounds__(256) void carry_kernel(float *entering, const float *steps, const float *A, int N, int C, int segments) {
  const int64_t i = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x, size = static_cast<int64_t>(N) * C;
  if (i >= size) return;
  const int n = static_cast<int>(i / C), c = static_cast<int>(i - static_cast<int64_t>(n) * C);
  const float A2 = A[static_cast<int64_t>(c) * N + n] * kLog2e;
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
    for (int k = 0; k < kAhead; ++k) out[k] = h = sum[k] < 0.f ? e[k] : fmaf(__builtin_amdgcn_exp2f(sum[k] * A2), h, e[k]);
    if (s0 + kAhead < segments - 1) request(s0 + kAhead);
#pragma unroll
    for (int k = 0; k < kAhead; ++k)
      if (s0 + k < segments - 1) entering[(s0 + k) * size + i] = out[k];
  }
}

__device__ __forceinline__ float value(float v) { return v; }
__device__ __forceinline__ float value(uint16_t v) { return bf16_bits_to_f32(v); }
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

// How a call is cut up.  Fewer states a wave make more waves, which share what is done once a token (step sizes, gates), wait at
// barriers, and read step sizes and inflows from LDS each.  16 states of 5120 channels, us by tokens, with 8 / 4 / 2 states a wave, each at
// its best segments: 512 tokens 41 / 39 / 42; 2048 95 / 99 / 111; 16384 545 / 655 / 776 (16 states: 537).  1536 channels: 61 tokens 16.3 / 14.0 /
// 12.7; 256 20.7 / 17.9 / 17.3; 2048 (fp32) 51 / 47 / 47.
struct Cut {
  int states, waves;         // a wave, for a channel
  int64_t most_segments;     // that the workspace has room for: never fewer for more tokens
  int segment;               // tokens
  int padded() const { return states * waves; }
};
Cut cut_of(const SelectiveDims &d) {
  int padded = 8;
  while (padded < d.N) padded *= 2;
  const int64_t groups = (d.C + 63) / 64, work = d.T * groups * padded / 16;  // of 16 states, tokens times waves
  Cut c = {};
  c.states = work >= 100000 ? 8 : work >= 20000 ? 4 : 2;
  if (c.states < padded / 8) c.states = padded / 8;
  c.waves = padded / c.states;
  // Segments make waves too, at the price of the states pass, and of their states' way through memory: some 16 waves a SIMD where
  // there is work for them, 5 where there is less.  Up to 80 tokens the three launches cost more than they save.
  const int64_t shortest = c.states >= 8 ? 48 : 32, waves = c.states >= 8 ? 16384 : 5120;
  c.most_segments = d.T <= 80 ? 1 : std::max<int64_t>(1, std::min((d.T + shortest - 1) / shortest, waves / c.waves / groups));
  const int64_t least = (d.T + c.most_segments - 1) / c.most_segments, block = block_of(c.waves);
  const int64_t wanted = knobs().selective_segment > 0 ? std::max<int64_t>(knobs().selective_segment, least) : least;
  c.segment = static_cast<int>((wanted + block - 1) / block * block);
  return c;
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

template <bool kIo, bool kDt, bool kBc, int NS, int W>
hipError_t launch_split(const ScanArgs &a, hipStream_t stream) {
  const unsigned groups = (a.d.C + 63) / 64;
  if (a.segments > 1) {
    hipLaunchKernelGGL((selective_kernel<kIo, kDt, kBc, NS, W, true>), dim3(groups, a.segments - 1), dim3(64 * W), 0, stream, a);
    if (const hipError_t e = hipGetLastError(); e != hipSuccess) return e;
    hipLaunchKernelGGL(carry_kernel, dim3(static_cast<unsigned>((static_cast<int64_t>(a.d.C) * a.d.N + 255) / 256)), dim3(256), 0, stream, a.entering, a.steps, a.a.A, a.d.N, a.d.C, a.segments);
    if (const hipError_t e = hipGetLastError(); e != hipSuccess) return e;
  }
  hipLaunchKernelGGL((selective_kernel<kIo, kDt, kBc, NS, W, false>), dim3(groups, a.segments), dim3(64 * W), 0, stream, a);
  return hipGetLastError();
}

template <bool kIo, bool kDt, bool kBc>
hipError_t launch_typed(const ScanArgs &a, const Cut &c, hipStream_t stream) {
  switch (c.states * 16 + c.waves) {
    case 8 * 16 + 1: return launch_split<kIo, kDt, kBc, 8, 1>(a, stream);
    case 4 * 16 + 2: return launch_split<kIo, kDt, kBc, 4, 2>(a, stream);
    case 2 * 16 + 4: return launch_split<kIo, kDt, kBc, 2, 4>(a, stream);
    case 8 * 16 + 2: return launch_split<kIo, kDt, kBc, 8, 2>(a, stream);
    case 4 * 16 + 4: return launch_split<kIo, kDt, kBc, 4, 4>(a, stream);
    case 2 * 16 + 8: return launch_split<kIo, kDt, kBc, 2, 8>(a, stream);
    case 8 * 16 + 4: return launch_split<kIo, kDt, kBc, 8, 4>(a, stream);
    case 4 * 16 + 8: return launch_split<kIo, kDt, kBc, 4, 8>(a, stream);
    case 8 * 16 + 8: return launch_split<kIo, kDt, kBc, 8, 8>(a, stream);
    case 16 * 16 + 8: return launch_split<kIo, kDt, kBc, 16, 8>(a, stream);
    case 32 * 16 + 8: return launch_split<kIo, kDt, kBc, 32, 8>(a, stream);
    default: return hipErrorInvalidValue;
  }
}

}  // namespace

// Whether no launch of a call has 2^32 threads or more.
bool selective_prefill_fits(const SelectiveDims &d) {
  const Cut c = cut_of(d);
  const int64_t groups = (d.C + 63) / 64;
  return c.most_segments <= 65535 && groups * c.most_segments * c.waves * 64 < (int64_t{1} << 32) &&
         (static_cast<int64_t>(d.T) + 256) * c.padded() < (int64_t{1} << 32);
}

size_t selective_prefill_workspace_bytes(const SelectiveDims &d) { return plan_of(d, cut_of(d)).total; }

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
  if (!d.bf16) return launch_typed<false, false, false>(a, s, stream);
  if (d.dt_bf16) return whole ? launch_typed<true, true, true>(a, s, stream) : launch_typed<true, true, false>(a, s, stream);
  return whole ? launch_typed<true, false, true>(a, s, stream) : launch_typed<true, false, false>(a, s, stream);
}

}  // namespace ssd
