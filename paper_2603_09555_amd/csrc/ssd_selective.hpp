// The selective state space scan (a decay of its own for every channel and state): what its translation units share.
#pragma once

#include "ssd_internal.hpp"

namespace ssd {

constexpr int kMostSelectiveStates = 256;

// Validated shape of a call.
struct SelectiveDims {
  int B, T, C, N;       // sequences, tokens of them all, channels, states of a channel
  bool bf16, dt_bf16;   // types of x, B, C, z, y; of dt
  DtXform dtx;
};

struct SelectiveArgs {
  const void *x, *dt, *B, *C, *z;  // z: or null
  const float *A, *D;              // D: or null
  int64_t b_stride, c_stride, z_stride;
  void *y;
};

constexpr float kLog2e = 1.4426950408889634f;
__device__ __forceinline__ float silu(float v) { return v * __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(v * -kLog2e)); }
// A state's decay in powers of two a unit of step size.  -inf, a state that keeps nothing, becomes the lowest finite value, which says
// the same of steps from 2^-120 on (2^(-2^8) is nothing in fp32).  A step of zero then leaves such a state as it is, like all others,
// where 0 x -inf would make it NaN: that is what steps driven to zero mean, and what the by-state kernel takes behind a sequence's end.
// A NaN stays one.
__device__ __forceinline__ float decay_rate(float A) {
  const float rate = A * kLog2e;
  return rate < -3.4028235e38f ? -3.4028235e38f : rate;
}
// softplus(v) = max(v, 0) + log(1 + e), e = exp(-|v|), in 18 issue slots of the vector unit, within 4 2^-24 of itself down to
// v = -80.  What rounding the exponent p = -|v| log2(e) takes away comes back as a factor of e, and what rounding 1 + e does, which is
// most of a small e, as the first term of the logarithm's series (1 / (1 + e) within 0.09 there, of something below 2^-24).
__device__ __forceinline__ float softplus(float v) {
  const float a = fmaxf(-fabsf(v), -100.f);  // (behind it e is nothing; a NaN comes back with max(v, 0))
  const float p = a * kLog2e, rest = fmaf(p, -0.693147182f, a);
  const float e2 = __builtin_amdgcn_exp2f(p), e = fmaf(e2, rest, e2);
  const float u = 1.f + e, lost = e - (u - 1.f);
  return (v <= 0.f ? 0.f : v) + fmaf(lost, fmaf(-0.5f, e, 1.f), __builtin_amdgcn_logf(u) * 0.693147182f);
}
// The step size of a raw value.
__device__ __forceinline__ float step_of(float v, float bias, const DtXform &map) {
  v += bias;
  if (map.softplus) v = softplus(v);
  return map.hi > 0.f ? fminf(fmaxf(v, map.lo), map.hi) : v;
}

bool selective_prefill_fits(const SelectiveDims &d);
size_t selective_prefill_workspace_bytes(const SelectiveDims &d);
hipError_t launch_selective_prefill(const SelectiveDims &d, const SelectiveArgs &a, const int32_t *cu, const float *h0, float *final_state,
                                    void *workspace, hipStream_t stream);
bool selective_step_fits(const SelectiveDims &d);
hipError_t launch_selective_step(const SelectiveDims &d, const SelectiveArgs &a, float *state, hipStream_t stream);

}  // namespace ssd
