// Attention of a query row by one wave: a lane holds four of the head's values and walks the tokens one by one.
#pragma once

#include "ssd_attn.hpp"

namespace ssd {

struct AttnArgs {
  const int32_t *cu, *lens, *table;
  const void *q, *k, *v;
  void *y;
  AttnDims d;
  float scale_log2;  // scale * log2(e)
};

template <bool kBf16>
__global__ __launch_bounds__(64) void attn_rows_kernel(const AttnArgs a) {
  using namespace block;
  using E = typename std::conditional<kBf16, uint16_t, float>::type;
  const int token = blockIdx.x, head = blockIdx.y, lane = threadIdx.x, c = 4 * lane;
  const Token at = find_token(a.d, a.cu, a.lens, token);
  if (!at.found) return;
  const int seq = at.seq, pos = at.pos;
  const bool mine = c < a.d.D;
  auto load4 = [&](const void *base, int64_t row, float v[4]) {
    const E *p = static_cast<const E *>(base) + row * a.d.D + c;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if (!mine) v[i] = 0.f;
      else if constexpr (kBf16) v[i] = __uint_as_float(static_cast<uint32_t>(p[i]) << 16);
      else v[i] = p[i];
    }
  };
  const int64_t row = static_cast<int64_t>(token) * a.d.H + head;
  float q[4], o[4] = {0.f, 0.f, 0.f, 0.f}, m = -3.0e38f, l = 0.f;
  load4(a.q, row, q);
  const int lo = a.d.window > 0 ? max(0, pos + 1 - a.d.window) : 0;
  for (int t = lo; t <= pos; ++t) {
    const int64_t slot = slot_of(a.d, a.table, seq, t, head / a.d.G);
    if (slot < 0) continue;
    float k[4], v[4];
    load4(a.k, slot, k);
    load4(a.v, slot, v);
    const float s = wave_sum(q[0] * k[0] + q[1] * k[1] + q[2] * k[2] + q[3] * k[3]) * a.scale_log2;
    const float top = fmaxf(m, s), keep = __builtin_amdgcn_exp2f(m - top), p = __builtin_amdgcn_exp2f(s - top);
    m = top;
    l = fmaf(l, keep, p);
#pragma unroll
    for (int i = 0; i < 4; ++i) o[i] = fmaf(o[i], keep, p * v[i]);
  }
  if (!mine) return;
  const float r = l > 0.f ? 1.f / l : (l == 0.f ? 0.f : l);
  E *y = static_cast<E *>(a.y) + row * a.d.D + c;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if constexpr (kBf16) y[i] = static_cast<uint16_t>(pack2(o[i] * r, 0.f));
    else y[i] = o[i] * r;
  }
}

inline hipError_t launch_attn_rows(const AttnDims &d, const int32_t *cu, const int32_t *lens, const int32_t *table, const void *q,
                                   const void *k, const void *v, float scale, void *y, hipStream_t stream) {
  const AttnArgs a = {cu, lens, table, q, k, v, y, d, scale * 1.44269504f};
  const dim3 grid(cu != nullptr ? d.T : d.B, d.H);
  if (d.bf16)
    hipLaunchKernelGGL(attn_rows_kernel<true>, grid, dim3(64), 0, stream, a);
  else
    hipLaunchKernelGGL(attn_rows_kernel<false>, grid, dim3(64), 0, stream, a);
  return hipGetLastError();
}

}  // namespace ssd
