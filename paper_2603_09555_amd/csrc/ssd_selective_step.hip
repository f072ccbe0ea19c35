// Selective state space scan of one new token of each sequence:
//
//   d = step(dt[b][c]),  h[b][c][n] = exp(d A[c][n]) h[b][c][n] + d x[b][c] B[b][n]
//   y[b][c] = (sum_n C[b][n] h[b][c][n] + D[c] x[b][c]) silu(z[b][c])
//
// Bound by one read and one write of the states.  A lane holds four neighbouring states of a channel (16 bytes), the next
// lanes the channel's others: sums over them stay within 4 lanes for 16 states, within 64 for 256.  Where there are many
// sequences a lane takes those states of two of them, which are on their way together, and reads the decays once.
//
// 256 sequences x 5120 channels x 16 states, bf16 or fp32: 36 us, 4.9 TB/s, where eight batches take turns, so that states come from
// memory; 30 where one batch's do, of which the last-level cache holds what it can.  (Inputs in turn, between the two: 35, and 44 with
// one sequence a lane.)  One sequence 4.3 us, the launch.
#include "ssd_selective.hpp"

namespace ssd {
namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint16_t u16x4 __attribute__((ext_vector_type(4)));

struct StepArgs {
  SelectiveArgs a;
  float *state;
  SelectiveDims d;
  int lanes;           // of a channel: a power of two, four states each
  unsigned across;     // workgroups a sequence
  uint32_t inv_across;
};

__device__ __forceinline__ float to_float(float v) { return v; }
__device__ __forceinline__ float to_float(uint16_t v) { return bf16_bits_to_f32(v); }
__device__ __forceinline__ void put(float *p, float v) { *p = v; }
__device__ __forceinline__ void put(uint16_t *p, float v) { *p = __builtin_bit_cast(uint16_t, static_cast<__bf16>(v)); }

// Four neighbouring values of `n` in a row, from `at` on, of which those behind the n-th are zeros.  kWhole: they are all there.
// Otherwise the last four of the row are taken where four from `at` are not there, and moved up.
__device__ __forceinline__ void raw4(const float *p, float v[4]) {
  const f32x4 q = *reinterpret_cast<const f32x4 __attribute__((aligned(4))) *>(p);
#pragma unroll
  for (int k = 0; k < 4; ++k) v[k] = q[k];
}
__device__ __forceinline__ void raw4(const uint16_t *p, float v[4]) {
  const u16x4 q = *reinterpret_cast<const u16x4 __attribute__((aligned(2))) *>(p);
#pragma unroll
  for (int k = 0; k < 4; ++k) v[k] = to_float(q[k]);
}
template <bool kWhole, typename E>
__device__ __forceinline__ void load4(const E *row, int at, int n, float v[4]) {
  if (kWhole) {
    raw4(row + at, v);
  } else if (n < 4) {
#pragma unroll
    for (int k = 0; k < 4; ++k) v[k] = at + k < n ? to_float(row[at + k]) : 0.f;
  } else {
    const int from = min(at, n - 4), by = at - from;
    raw4(row + from, v);
    if (by >= 2) {
      v[0] = v[2];
      v[1] = v[3];
    }
    if (by & 1) {
      v[0] = v[1];
      v[1] = v[2];
      v[2] = v[3];
    }
#pragma unroll
    for (int k = 0; k < 4; ++k) v[k] = at + k < n ? v[k] : 0.f;
  }
}

// kWhole: as many states as four times the lanes.  R: sequences a lane.
template <typename E, typename EDt, bool kWhole, int R>
__global__ __launch_bounds__(256) void selective_step_kernel(const StepArgs a) {
  const int lanes = a.lanes, N = a.d.N, C = a.d.C;
  const int row = quotient(blockIdx.x, a.across, a.inv_across), b0 = row * R;
  const int i = static_cast<int>(blockIdx.x - row * a.across) * 256 + static_cast<int>(threadIdx.x);
  const int c_real = i / lanes, piece = i & (lanes - 1), first = 4 * piece;
  const int c = min(c_real, C - 1);
  const bool there = c_real < C && first < N;
  float A2[4], h[R][4], Bv[R][4], Cv[R][4], x[R], dt[R], z[R];
  load4<kWhole>(a.a.A + static_cast<int64_t>(c) * N, first, N, A2);
#pragma unroll
  for (int r = 0; r < R; ++r) {
    const int b = min(b0 + r, a.d.B - 1);  // (surplus ones: the last sequence, not written)
    const int64_t channel = static_cast<int64_t>(b) * C + c;
    load4<kWhole>(a.state + channel * N, first, N, h[r]);
    load4<kWhole>(static_cast<const E *>(a.a.B) + b * a.a.b_stride, first, N, Bv[r]);
    load4<kWhole>(static_cast<const E *>(a.a.C) + b * a.a.c_stride, first, N, Cv[r]);
    x[r] = to_float(static_cast<const E *>(a.a.x)[channel]);
    dt[r] = to_float(static_cast<const EDt *>(a.a.dt)[channel]);
    z[r] = a.a.z ? to_float(static_cast<const E *>(a.a.z)[b * a.a.z_stride + c]) : 0.f;
  }
  const float bias = a.d.dtx.bias ? a.d.dtx.bias[c] : 0.f, skip = a.a.D ? a.a.D[c] : 0.f;
#pragma unroll
  for (int k = 0; k < 4; ++k) A2[k] = decay_rate(A2[k]);
#pragma unroll
  for (int r = 0; r < R; ++r) {
    const float d = step_of(dt[r], bias, a.d.dtx), u = d * x[r];
    float sum = 0.f;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      h[r][k] = fmaf(__builtin_amdgcn_exp2f(d * A2[k]), h[r][k], u * Bv[r][k]);
      sum = fmaf(Cv[r][k], h[r][k], sum);
    }
    for (int k = 1; k < lanes; k <<= 1) sum += __shfl_xor(sum, k);
    if (!there || b0 + r >= a.d.B) continue;
    const int64_t channel = static_cast<int64_t>(b0 + r) * C + c;
    float *const state = a.state + channel * N + first;
    if (kWhole) {
      *reinterpret_cast<f32x4 *>(state) = f32x4{h[r][0], h[r][1], h[r][2], h[r][3]};
    } else {
#pragma unroll
      for (int k = 0; k < 4; ++k)
        if (first + k < N) state[k] = h[r][k];
    }
    if (piece == 0) {
      sum = fmaf(skip, x[r], sum);
      if (a.a.z) sum *= silu(z[r]);
      put(static_cast<E *>(a.a.y) + channel, sum);
    }
  }
}

int lanes_of(int N) {
  int l = 1;
  while (4 * l < N) l <<= 1;
  return l;
}
int64_t across_of(const SelectiveDims &d) { return (static_cast<int64_t>(d.C) * lanes_of(d.N) + 255) / 256; }
// Sequences a lane: two, as long as that leaves workgroups for all CUs.
int sequences_of(const SelectiveDims &d) { return d.B * across_of(d) >= 4096 ? 2 : 1; }

template <typename E, typename EDt, bool kWhole>
void launch_rows(const StepArgs &a, int rows, hipStream_t stream) {
  const dim3 grid(static_cast<unsigned>((a.d.B + int64_t{rows} - 1) / rows * a.across));
  if (rows == 2)
    hipLaunchKernelGGL((selective_step_kernel<E, EDt, kWhole, 2>), grid, dim3(256), 0, stream, a);
  else
    hipLaunchKernelGGL((selective_step_kernel<E, EDt, kWhole, 1>), grid, dim3(256), 0, stream, a);
}
template <typename E, typename EDt>
void launch_typed(const StepArgs &a, int rows, hipStream_t stream) {
  if (a.d.N == 4 * a.lanes) launch_rows<E, EDt, true>(a, rows, stream);
  else launch_rows<E, EDt, false>(a, rows, stream);
}

}  // namespace

bool selective_step_fits(const SelectiveDims &d) { return (d.B + int64_t{sequences_of(d)} - 1) / sequences_of(d) * across_of(d) < (1 << 24); }

hipError_t launch_selective_step(const SelectiveDims &d, const SelectiveArgs &args, float *state, hipStream_t stream) {
  StepArgs a = {args, state, d, lanes_of(d.N), static_cast<unsigned>(across_of(d)), 0};
  a.inv_across = inverse_of(static_cast<int>(a.across));
  const int rows = sequences_of(d);
  if (!d.bf16) launch_typed<float, float>(a, rows, stream);
  else if (d.dt_bf16) launch_typed<uint16_t, uint16_t>(a, rows, stream);
  else launch_typed<uint16_t, float>(a, rows, stream);
  return hipGetLastError();
}

}  // namespace ssd
