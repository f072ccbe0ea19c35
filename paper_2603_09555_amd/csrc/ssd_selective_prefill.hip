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

#include "ssd_selective.hpp"

namespace ssd {
namespace {

constexpr float kLog2e = 1.4426950408889634f;

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

__device__ __forceinline__ float silu(float v) { return v * __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(v * -kLog2e)); }

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

template <bool kBf16>
struct Io;
template <>
struct Io<true> {
  typedef uint16_t type;
};
template <>
struct Io<false> {
  typedef float type;
};
__device__ __forceinline__ float to_float(float v) { return v; }
__device__ __forceinline__ float to_float(uint16_t v) { return bf16_bits_to_f32(v); }
__device__ __forceinline__ void put(float *p, float v) { *p = v; }
__device__ __forceinline__ void put(uint16_t *p, float v) { *p = __builtin_bit_cast(uint16_t, static_cast<__bf16>(v)); }

// kIo, kDt, kBc: bf16 (x, z, y; dt; rows of B and C).  NS states a wave, W waves for a channel's states; a block of tokens is
// kBlock.  kStates: the states pass.
template <bool kIo, bool kDt, bool kBc, int NS, int W, bool kStates>
__global__ __launch_bounds__(64 * W) void selective_kernel(const ScanArgs a) {
  using E = typename Io<kIo>::type;
  using EDt = typename Io<kDt>::type;
  constexpr int kBlock = 8, kOwn = W > kBlock ? 1 : kBlock / W;  // tokens of a block; those that a wave prepares and finishes
  static_assert(kBlock % W == 0, "a wave's tokens are as many as any other's");
  __shared__ float lds_d[W > 1 ? kBlock : 1][64], lds_u[W > 1 ? kBlock : 1][64], lds_part[W > 1 && !kStates ? W : 1][W > 1 ? kBlock : 1][64];
  const int lane = threadIdx.x & 63, wave = W > 1 ? __builtin_amdgcn_readfirstlane(threadIdx.x / 64) : 0;
  const int n0 = wave * NS;
  const int N = a.d.N, C = a.d.C, T = a.d.T;
  const int c_real = blockIdx.x * 64 + lane, c = min(c_real, C - 1);
  const bool live = c_real < C;
  const int s = blockIdx.y;
  const int t0 = s * a.segment, t1 = min(T, t0 + a.segment);

  float A2[NS], h[NS];
#pragma unroll
  for (int n = 0; n < NS; ++n) A2[n] = n0 + n < N ? a.a.A[static_cast<int64_t>(c) * N + n0 + n] * kLog2e : 0.f;
  const float bias = a.d.dtx.bias ? a.d.dtx.bias[c] : 0.f, skip = !kStates && a.a.D ? a.a.D[c] : 0.f;
  const E *const x = static_cast<const E *>(a.a.x) + c;
  const EDt *const dt = static_cast<const EDt *>(a.a.dt) + c;
  const E *const z = kStates || !a.a.z ? nullptr : static_cast<const E *>(a.a.z) + c;
  E *const y = static_cast<E *>(a.a.y) + c;
  float total = 0.f;  // of the step sizes

  auto load_state = [&](const float *from, int64_t stride) {  // states n0.. of this lane's channel, `stride` apart
#pragma unroll
    for (int n = 0; n < NS; ++n) h[n] = n0 + n < N && from ? from[(n0 + n) * stride] : 0.f;
  };
  auto store_state = [&](float *to, int64_t stride) {
#pragma unroll
    for (int n = 0; n < NS; ++n)
      if (n0 + n < N && live) to[(n0 + n) * stride] = h[n];
  };

  // tokens [from, to), which are of one sequence
  auto walk = [&](int from, int to) {
    if (from >= to) return;
    struct Raw {
      E x[kOwn], z[kOwn];
      EDt dt[kOwn];
    } raw;
    auto request = [&](int tb) {
#pragma unroll
      for (int i = 0; i < kOwn; ++i) {
        const int64_t t = min(tb + wave * kOwn + i, to - 1);  // (surplus ones: the last row)
        raw.x[i] = x[t * C];
        raw.dt[i] = dt[t * C];
        if (z) raw.z[i] = z[t * a.a.z_stride];
      }
    };
    request(from);
    for (int tb = from; tb < to; tb += kBlock) {
      const Raw now = raw;
      if (tb + kBlock < to) request(tb + kBlock);
      float d_own[kOwn], u_own[kOwn];
#pragma unroll
      for (int i = 0; i < kOwn; ++i) {
        d_own[i] = dt_apply_branchless(to_float(now.dt[i]), bias, a.d.dtx);
        u_own[i] = d_own[i] * to_float(now.x[i]);
        if constexpr (W > 1) {
          lds_d[wave * kOwn + i][lane] = d_own[i];
          lds_u[wave * kOwn + i][lane] = u_own[i];
        }
      }
      if constexpr (W > 1) __syncthreads();
      float sum[kBlock];
#pragma unroll
      for (int i = 0; i < kBlock; ++i) {
        if (tb + i >= to) break;
        const float d = W > 1 ? lds_d[i][lane] : d_own[i % kOwn], u = W > 1 ? lds_u[i][lane] : u_own[i % kOwn];
        Uniform<kBc, NS> bt, ct;
        const int64_t t = tb + i;
        constexpr int kSize = kBc ? 2 : 4;
        bt.load(static_cast<const char *>(a.rows.b) + (t * a.rows.b_stride + n0) * kSize);
        if constexpr (!kStates) ct.load(static_cast<const char *>(a.rows.c) + (t * a.rows.c_stride + n0) * kSize);
        if constexpr (kStates) total += d;
        float acc = 0.f;
#pragma unroll
        for (int n = 0; n < NS; ++n) {
          h[n] = fmaf(__builtin_amdgcn_exp2f(d * A2[n]), h[n], u * bt.of(n));
          if constexpr (!kStates) acc = fmaf(ct.of(n), h[n], acc);
        }
        sum[i] = acc;
        if constexpr (W > 1 && !kStates) lds_part[wave][i][lane] = acc;
      }
      if constexpr (W > 1) __syncthreads();
      if constexpr (!kStates) {
#pragma unroll
        for (int i = 0; i < kOwn; ++i) {
          const int t = tb + wave * kOwn + i;
          if (t >= to) break;
          float v;
          if constexpr (W > 1) {
            v = lds_part[0][wave * kOwn + i][lane];
#pragma unroll
            for (int w = 1; w < W; ++w) v += lds_part[w][wave * kOwn + i][lane];
          } else {
            v = sum[i];
          }
          v = fmaf(skip, to_float(now.x[i]), v);
          if (z) v *= silu(to_float(now.z[i]));
          if (live) put(y + static_cast<int64_t>(t) * C, v);
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

// The state that enters each segment but the first, in place of the one at the end of the segment before.
__global__ __launch_bounds__(256) void carry_kernel(float *entering, const float *steps, const float *A, int N, int C, int segments) {
  const int c = blockIdx.x * 256 + threadIdx.x, n = blockIdx.y;
  if (c >= C) return;
  const float A2 = A[static_cast<int64_t>(c) * N + n] * kLog2e;
  float h = 0.f;
  for (int s = 0; s < segments - 1; ++s) {
    float *const at = entering + (static_cast<int64_t>(s) * N + n) * C + c;
    const float sum = steps[static_cast<int64_t>(s) * C + c], e = *at;
    h = sum < 0.f ? e : fmaf(__builtin_amdgcn_exp2f(sum * A2), h, e);
    *at = h;
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
  out[i] = n < N ? to_float(static_cast<const E *>(b)[t * b_stride + n]) : 0.f;
  out[values + i] = n < N ? to_float(static_cast<const E *>(c)[t * c_stride + n]) : 0.f;
}

// States a wave, waves for a channel's.
struct Split {
  int states, waves;
  int padded() const { return states * waves; }
};
Split split_of(int N) {
  if (N <= 8) return {8, 1};
  if (N <= 16) return {16, 1};
  if (N <= 32) return {16, 2};
  if (N <= 64) return {16, 4};
  if (N <= 128) return {32, 4};
  return {32, 8};
}

int segment_of(const SelectiveDims &d) {
  (void)d;
  return 1 << 30;
}
int64_t segments_of(const SelectiveDims &d) { return (static_cast<int64_t>(d.T) + segment_of(d) - 1) / segment_of(d); }

// Parts of the workspace, in bytes.
struct Plan {
  size_t rows, entering, steps, begun, total;
};
Plan plan_of(const SelectiveDims &d) {
  Plan p = {};
  const size_t segments = static_cast<size_t>(segments_of(d));
  size_t at = 0;
  const auto take = [&](size_t bytes) {
    const size_t was = at;
    at += round_up(bytes, 256);
    return was;
  };
  p.rows = take(static_cast<size_t>(d.T) * 2 * split_of(d.N).padded() * 4);
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
    hipLaunchKernelGGL(carry_kernel, dim3((a.d.C + 255) / 256, a.d.N), dim3(256), 0, stream, a.entering, a.steps, a.a.A, a.d.N, a.d.C, a.segments);
    if (const hipError_t e = hipGetLastError(); e != hipSuccess) return e;
  }
  hipLaunchKernelGGL((selective_kernel<kIo, kDt, kBc, NS, W, false>), dim3(groups, a.segments), dim3(64 * W), 0, stream, a);
  return hipGetLastError();
}

template <bool kIo, bool kDt, bool kBc>
hipError_t launch_typed(const ScanArgs &a, const Split &s, hipStream_t stream) {
  if (s.states == 8) return launch_split<kIo, kDt, kBc, 8, 1>(a, stream);
  if (s.states == 16 && s.waves == 1) return launch_split<kIo, kDt, kBc, 16, 1>(a, stream);
  if (s.states == 16 && s.waves == 2) return launch_split<kIo, kDt, kBc, 16, 2>(a, stream);
  if (s.states == 16) return launch_split<kIo, kDt, kBc, 16, 4>(a, stream);
  if (s.waves == 4) return launch_split<kIo, kDt, kBc, 32, 4>(a, stream);
  return launch_split<kIo, kDt, kBc, 32, 8>(a, stream);
}

}  // namespace

// Whether no launch of a call has 2^32 threads or more.
bool selective_prefill_fits(const SelectiveDims &d) {
  const Split s = split_of(d.N);
  const int64_t groups = (d.C + 63) / 64, segments = segments_of(d);
  return segments <= 65535 && groups * segments * s.waves * 64 < (int64_t{1} << 32) && (static_cast<int64_t>(d.T) + 256) * s.padded() < (int64_t{1} << 32);
}

size_t selective_prefill_workspace_bytes(const SelectiveDims &d) { return std::max<size_t>(plan_of(d).total, 256); }

hipError_t launch_selective_prefill(const SelectiveDims &d, const SelectiveArgs &args, const int32_t *cu, const float *h0, float *final_state,
                                    void *workspace, hipStream_t stream) {
  const Plan p = plan_of(d);
  const Split s = split_of(d.N);
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
  a.segment = segment_of(d);
  a.segments = static_cast<int>(segments_of(d));
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
