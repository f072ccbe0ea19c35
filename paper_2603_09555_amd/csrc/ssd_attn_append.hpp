// What the two kernels that append to a paged cache share: without norms (ssd_attn_append.hip) and with (ssd_attn_append_norm.hip).
#pragma once

#include "ssd_attn.hpp"

namespace ssd {
namespace {

using namespace block;

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

}  // namespace
}  // namespace ssd
