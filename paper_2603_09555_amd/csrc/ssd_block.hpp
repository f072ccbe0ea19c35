// What the operators of a hybrid stack's other layers share: norms, and attention over a paged cache.
#pragma once

#include "ssd_internal.hpp"

namespace ssd {
namespace block {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

__device__ __forceinline__ uint32_t pack2(float lo, float hi) {  // two fp32 -> packed bf16, RNE
  typedef float f32x2 __attribute__((ext_vector_type(2)));
  typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
  const f32x2 v = {lo, hi};
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(v, bf16x2));
}
__device__ __forceinline__ float bf_lo(uint32_t u) { return __uint_as_float(u << 16); }
__device__ __forceinline__ float bf_hi(uint32_t u) { return __uint_as_float(u & 0xffff0000u); }

// Eight neighbouring values, of which the first `left` exist (eight if more).  Addresses need no more than the element's
// alignment: rows of odd widths begin anywhere, and gfx950's global accesses of 16 bytes may as well.
struct Bf16 {
  typedef uint16_t type;
  typedef u32x4 __attribute__((aligned(2))) vec;
  static __device__ __forceinline__ void load(const uint16_t *p, int left, float v[8]) {
    if (left >= 8) {
      const u32x4 q = *reinterpret_cast<const vec *>(p);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        v[2 * i] = bf_lo(q[i]);
        v[2 * i + 1] = bf_hi(q[i]);
      }
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] = i < left ? __uint_as_float(static_cast<uint32_t>(p[i]) << 16) : 0.f;
    }
  }
  static __device__ __forceinline__ void store(uint16_t *p, int left, const float v[8]) {
    u32x4 q;
#pragma unroll
    for (int i = 0; i < 4; ++i) q[i] = pack2(v[2 * i], v[2 * i + 1]);
    if (left >= 8) {
      *reinterpret_cast<vec *>(p) = q;
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (i < left) p[i] = static_cast<uint16_t>(q[i / 2] >> (16 * (i & 1)));
    }
  }
};
struct F32 {
  typedef float type;
  typedef f32x4 __attribute__((aligned(4))) vec;
  static __device__ __forceinline__ void load(const float *p, int left, float v[8]) {
    if (left >= 8) {
      const f32x4 a = *reinterpret_cast<const vec *>(p), b = *reinterpret_cast<const vec *>(p + 4);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        v[i] = a[i];
        v[i + 4] = b[i];
      }
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] = i < left ? p[i] : 0.f;
    }
  }
  static __device__ __forceinline__ void store(float *p, int left, const float v[8]) {
    if (left >= 8) {
      f32x4 a, b;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        a[i] = v[i];
        b[i] = v[i + 4];
      }
      *reinterpret_cast<vec *>(p) = a;
      *reinterpret_cast<vec *>(p + 4) = b;
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (i < left) p[i] = v[i];
    }
  }
};

// v / (1 + exp(-v)) with the hardware exp2 and reciprocal (each within 1 ulp): an IEEE division per element would make a
// stream ALU bound.
__device__ __forceinline__ float silu(float v) {
  return v * __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(v * -1.4426950408889634f));
}

}  // namespace block

// Validated shape of an attention call.
struct AttnDims {
  int B, T, H, Hk, D, G;   // sequences, new tokens, heads, key heads, headdim, H / Hk
  int npages, lg_page, max_pages;
  int window;              // 0 = no limit, otherwise smaller than capacity()
  bool bf16;
  __host__ __device__ int capacity() const { return max_pages << lg_page; }  // tokens of a sequence, at most 2^30
};

struct Rope {
  const float *cos, *sin;
  int half;                // pairs; 0 = no rotation
  int interleaved;
};

hipError_t launch_norm_gated(int64_t rows, int width, int groups, bool bf16, const void *y, const void *z, int64_t z_stride,
                             const float *weight, float eps, bool norm_first, void *out, hipStream_t stream);
hipError_t launch_norm_residual(int64_t rows, int width, bool bf16, bool stream_bf16, const void *x, const void *residual,
                                float scale, const float *weight, float eps, void *out, void *residual_out, hipStream_t stream);
// Whether the launches of an attention call of this shape have less than 2^32 threads each, which is what a launch takes.
constexpr int64_t kMostWorkgroups256 = (int64_t{1} << 24) - 1;  // of 256 threads
bool attn_append_fits(const AttnDims &d, bool queries);
bool attn_step_fits(const AttnDims &d);
bool attn_prefill_fits(const AttnDims &d);
hipError_t launch_attn_append(const AttnDims &d, const Rope &rope, const int32_t *cu, const int32_t *lens, const int32_t *table,
                              const void *q, int64_t q_stride, const void *k, int64_t k_stride, const void *v, int64_t v_stride,
                              void *q_out, void *k_cache, void *v_cache, hipStream_t stream);
// What a call uses of its workspace; what no call of fewer sequences and tokens, otherwise the same, uses more of.
size_t attn_step_used_bytes(const AttnDims &d);
size_t attn_step_workspace_bytes(const AttnDims &d);
hipError_t launch_attn_step(const AttnDims &d, const int32_t *lens, const int32_t *table, const void *q, const void *k_cache,
                            const void *v_cache, float scale, void *y, void *workspace, hipStream_t stream);
size_t attn_prefill_used_bytes(const AttnDims &d);
size_t attn_prefill_workspace_bytes(const AttnDims &d);
hipError_t launch_attn_prefill(const AttnDims &d, const int32_t *cu, const int32_t *lens, const int32_t *table, const void *q,
                               const void *k_cache, const void *v_cache, float scale, void *y, void *workspace,
                               hipStream_t stream);

}  // namespace ssd
