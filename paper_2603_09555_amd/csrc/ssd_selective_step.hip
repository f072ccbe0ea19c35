// Selective state space scan of one new token of each sequence:
//
//   d = step(dt[b][c]),  h[b][c][n] = exp(d A[c][n]) h[b][c][n] + d x[b][c] B[b][n]
//   y[b][c] = (sum_n C[b][n] h[b][c][n] + D[c] x[b][c]) silu(z[b][c])
//
// Bound by one read and one write of the states.  A lane holds four neighbouring states of a channel (16 bytes), the next
// lanes the channel's others: sums over them stay within 4 lanes for 16 states, within 64 for 256.
#include "ssd_selective.hpp"

namespace ssd {
namespace {

constexpr float kLog2e = 1.4426950408889634f;
typedef float f32x4 __attribute__((ext_vector_type(4)));

struct StepArgs {
  SelectiveArgs a;
  float *state;
  SelectiveDims d;
  int lanes;  // of a channel: a power of two, four states each
};

__device__ __forceinline__ float to_float(float v) { return v; }
__device__ __forceinline__ float to_float(uint16_t v) { return bf16_bits_to_f32(v); }
__device__ __forceinline__ void put(float *p, float v) { *p = v; }
__device__ __forceinline__ void put(uint16_t *p, float v) { *p = __builtin_bit_cast(uint16_t, static_cast<__bf16>(v)); }

template <typename E, typename EDt>
__global__ __launch_bounds__(256) void selective_step_kernel(const StepArgs a) {
  const int lanes = a.lanes, N = a.d.N, C = a.d.C;
  const int b = blockIdx.y;
  const int64_t i = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x;
  const int64_t c64 = i / lanes;
  const int piece = static_cast<int>(i) & (lanes - 1), first = 4 * piece;
  const bool there = c64 < C;
  const int c = there ? static_cast<int>(c64) : C - 1;
  const int64_t at = static_cast<int64_t>(b) * C + c;
  const int left = N - first;  // states from `first` on
  float A2[4], h[4], Bv[4], Cv[4];
  float *const state = a.state + at * N + first;
  const float *const A = a.a.A + static_cast<int64_t>(c) * N + first;
  const E *const Br = static_cast<const E *>(a.a.B) + b * a.a.b_stride + first, *const Cr = static_cast<const E *>(a.a.C) + b * a.a.c_stride + first;
  const bool whole = N % 4 == 0;
  if (whole && left > 0) {
    const f32x4 v = *reinterpret_cast<const f32x4 *>(state), w = *reinterpret_cast<const f32x4 *>(A);
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      h[k] = v[k];
      A2[k] = w[k] * kLog2e;
      Bv[k] = to_float(Br[k]);
      Cv[k] = to_float(Cr[k]);
    }
  } else {
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      h[k] = k < left ? state[k] : 0.f;
      A2[k] = k < left ? A[k] * kLog2e : 0.f;
      Bv[k] = k < left ? to_float(Br[k]) : 0.f;
      Cv[k] = k < left ? to_float(Cr[k]) : 0.f;
    }
  }
  const float x = to_float(static_cast<const E *>(a.a.x)[at]);
  const float d = dt_apply_branchless(to_float(static_cast<const EDt *>(a.a.dt)[at]), a.d.dtx.bias ? a.d.dtx.bias[c] : 0.f, a.d.dtx);
  const float u = d * x;
  float acc = 0.f;
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    h[k] = fmaf(__builtin_amdgcn_exp2f(d * A2[k]), h[k], u * Bv[k]);
    acc = fmaf(Cv[k], h[k], acc);
  }
  for (int k = 1; k < lanes; k <<= 1) acc += __shfl_xor(acc, k);
  if (!there) return;
  if (whole && left > 0) {
    *reinterpret_cast<f32x4 *>(state) = f32x4{h[0], h[1], h[2], h[3]};
  } else {
#pragma unroll
    for (int k = 0; k < 4; ++k)
      if (k < left) state[k] = h[k];
  }
  if (piece == 0) {
    acc = fmaf(a.a.D ? a.a.D[c] : 0.f, x, acc);
    if (a.a.z) {
      const float v = to_float(static_cast<const E *>(a.a.z)[b * a.a.z_stride + c]);
      acc *= v * __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(v * -kLog2e));
    }
    put(static_cast<E *>(a.a.y) + at, acc);
  }
}

int lanes_of(int N) {
  int l = 1;
  while (4 * l < N) l <<= 1;
  return l;
}

}  // namespace

bool selective_step_fits(const SelectiveDims &d) { return static_cast<int64_t>(d.B) * ((static_cast<int64_t>(d.C) * lanes_of(d.N) + 255) / 256) * 256 < (int64_t{1} << 32) && d.B <= 65535; }

hipError_t launch_selective_step(const SelectiveDims &d, const SelectiveArgs &args, float *state, hipStream_t stream) {
  StepArgs a = {args, state, d, lanes_of(d.N)};
  const dim3 grid(static_cast<unsigned>((static_cast<int64_t>(d.C) * a.lanes + 255) / 256), d.B);
  if (!d.bf16)
    hipLaunchKernelGGL((selective_step_kernel<float, float>), grid, dim3(256), 0, stream, a);
  else if (d.dt_bf16)
    hipLaunchKernelGGL((selective_step_kernel<uint16_t, uint16_t>), grid, dim3(256), 0, stream, a);
  else
    hipLaunchKernelGGL((selective_step_kernel<uint16_t, float>), grid, dim3(256), 0, stream, a);
  return hipGetLastError();
}

}  // namespace ssd
