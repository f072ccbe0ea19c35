// What the kernels of the depthwise convolution share: the batched prompts and the step (ssd_conv.hip), packed prompts
// (ssd_conv_varlen.hip).
#pragma once

#include "ssd_internal.hpp"

namespace ssd {
namespace {

constexpr int kConvThreads = 256;
constexpr int kRunMin = 16, kRunMax = 192;  // tokens per thread in the prefill kernel: chosen per launch

// SiLU v / (1 + exp(-v)) with the hardware exp2 and reciprocal (each within 1 ulp): the kernels are
// streams, and an IEEE division per element would make them ALU bound.
__device__ __forceinline__ float act_apply(float v, int act) {
  if (act != 1) return v;
  const float e = __builtin_amdgcn_exp2f(v * -1.4426950408889634f);
  return v * __builtin_amdgcn_rcpf(1.f + e);
}
typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));
typedef float f32x2_t __attribute__((ext_vector_type(2)));
__device__ __forceinline__ uint32_t pack_bf16x2(float lo, float hi) {  // two fp32 -> packed bf16, RNE
  f32x2_t v = {lo, hi};
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(v, bf16x2_t));
}

struct ConvOut {
  void *ptr[3];  // dense (batch, T, width[i]) tensors
  int begin[4];  // channel ranges [begin[i], begin[i+1])
};

// Output address of channel c (c is a multiple of VEC and ranges are multiples of VEC).
template <typename Io>
__device__ __forceinline__ typename Io::type *out_ptr(const ConvOut &o, size_t row, int c) {
  const int part = c >= o.begin[2] ? 2 : (c >= o.begin[1] ? 1 : 0);
  const int width = o.begin[part + 1] - o.begin[part];
  return static_cast<typename Io::type *>(o.ptr[part]) + row * width + (c - o.begin[part]);
}

// Tokens per thread: long runs amortise the k-1 rows a thread reads in front of its own and the
// weights it loads, but the threads should also fill the chip a whole number of times: the length in
// [shortest, kRunMax] with the least (rounds of waves) x (rows read per run).  `blocks_per_cu` is what the
// runtime reports for the kernel (its register count decides it).
int choose_run(int T, size_t groups_total, int ksize, int blocks_per_cu, int shortest = kRunMin) {
  const double slots = 256.0 * blocks_per_cu * kConvThreads;  // threads resident at once
  int best = shortest;
  double best_cost = 0.0;
  for (int len = shortest; len <= kRunMax; ++len) {
    const double runs = (T + len - 1) / len;
    const double rounds = static_cast<double>(static_cast<long long>((runs * groups_total + slots - 1) / slots));
    const double cost = rounds * (len + ksize - 1 + 4);  // + about four rows' worth of start-up per thread
    if (len == shortest || cost < best_cost) {
      best = len;
      best_cost = cost;
    }
  }
  return best;
}

ConvOut make_out(void *const z[3], const int width[3]) {
  ConvOut o;
  int c = 0;
  for (int i = 0; i < 3; ++i) {
    o.ptr[i] = z[i];
    o.begin[i] = c;
    c += width[i];
  }
  o.begin[3] = c;
  return o;
}

}  // namespace
}  // namespace ssd

#define SSD_CONV_DISPATCH(FN, ...)                                         \
  switch (ksize) {                                                         \
    case 2: return bf16 ? FN<IoBf16, 2>(__VA_ARGS__) : FN<IoF32, 2>(__VA_ARGS__); \
    case 3: return bf16 ? FN<IoBf16, 3>(__VA_ARGS__) : FN<IoF32, 3>(__VA_ARGS__); \
    case 4: return bf16 ? FN<IoBf16, 4>(__VA_ARGS__) : FN<IoF32, 4>(__VA_ARGS__); \
    case 5: return bf16 ? FN<IoBf16, 5>(__VA_ARGS__) : FN<IoF32, 5>(__VA_ARGS__); \
    case 6: return bf16 ? FN<IoBf16, 6>(__VA_ARGS__) : FN<IoF32, 6>(__VA_ARGS__); \
    case 7: return bf16 ? FN<IoBf16, 7>(__VA_ARGS__) : FN<IoF32, 7>(__VA_ARGS__); \
    case 8: return bf16 ? FN<IoBf16, 8>(__VA_ARGS__) : FN<IoF32, 8>(__VA_ARGS__); \
    default: return hipErrorInvalidValue;                                  \
  }
