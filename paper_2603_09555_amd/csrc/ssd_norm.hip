// The norms on either side of a Mamba-2 block:
//
//   gated, gate first:   u = y silu(z),  out = u rsqrt(mean(u^2) + eps) w
//   gated, norm first:   out = y rsqrt(mean(y^2) + eps) w silu(z)
//   residual:            r = residual + scale x,  residual_out = r,  out = r rsqrt(mean(r^2) + eps) w
//
// A unit -- a row, or one group of a row -- is read once, kept in registers as fp32 while its squares are summed, and written
// once.  A thread owns pieces of 8 neighbouring values (bf16: 16 bytes; fp32: 32).  Both are streams; with few rows they are a
// chain of two memory latencies and a reduction, and the unit is spread over as many threads as it has pieces for.
// 16384 rows of 5120, gated, bf16: 100 us, 5.0 TB/s (a copy: 4.9), fp32: 183 us, 5.5; 16383 of 768, residual, fp32: 40 us, 5.0; 16384 of
// 2560, bf16 on an fp32 stream: 95 us, 5.3, on a bf16 one: 66 us, 5.1; one row: 3 us, a launch.
#include <algorithm>

#include "ssd_block.hpp"

namespace ssd {
namespace {

using namespace block;

constexpr int kPiece = 8;
constexpr int kFewUnits = 512;
constexpr int64_t kMostThreads = int64_t{1} << 31;  // of a launch, which takes less than 2^32

enum Mode { kGateFirst = 0, kNormFirst = 1, kResidual = 2 };

struct NormArgs {
  const void *in;        // y or x
  const void *side;      // z or residual (nullptr: zeros)
  const float *weight;
  void *out;
  void *side_out;        // residual_out
  int64_t units, first;  // units; the first one of this launch
  int64_t side_stride;   // of z, in elements
  int width, n;          // values in a row, and in a unit
  int groups;
  float scale, eps, inv_n;
};

// What a piece becomes before the norm (v), and the factor it gets behind it (g; norm first only).
template <int kMode>
__device__ __forceinline__ void combine(float v[kPiece], float s[kPiece], float scale) {
#pragma unroll
  for (int i = 0; i < kPiece; ++i) {
    if (kMode == kResidual) {
      v[i] = fmaf(scale, v[i], s[i]);
    } else {
      s[i] = silu(s[i]);
      if (kMode == kGateFirst) v[i] *= s[i];
    }
  }
}

// kThreads threads a unit, kHold pieces a thread in registers (0: units too wide for that are read a second time, from the
// caches).  Units of a wave or less share a workgroup of four waves.
// The sum is that of runs of 64 pieces, added up in their order, whatever the number of threads: it does not depend on how many
// units there are, by which that number is chosen.
template <typename Io, typename Side, int kMode, int kThreads, int kHold>
__global__ __launch_bounds__(kThreads < 256 ? 256 : kThreads) void norm_kernel(const NormArgs a) {
  constexpr int kBlock = kThreads < 256 ? 256 : kThreads, kUnits = kBlock / kThreads, kWaves = kThreads < 64 ? 1 : kThreads / 64;
  const int t = threadIdx.x % kThreads;
  const int64_t unit = a.first + static_cast<int64_t>(blockIdx.x) * kUnits + threadIdx.x / kThreads;
  if (unit >= a.units) return;  // (all threads of a unit; workgroups of several waves a unit have one unit)
  int64_t row = unit;
  int first = 0;
  if (a.groups > 1) {
    row = static_cast<uint32_t>(unit) / static_cast<uint32_t>(a.groups);
    first = static_cast<int>(unit - row * a.groups) * a.n;
  }
  const typename Io::type *in = static_cast<const typename Io::type *>(a.in) + row * a.width + first;
  typename Io::type *out = static_cast<typename Io::type *>(a.out) + row * a.width + first;
  const typename Side::type *side = a.side == nullptr ? nullptr : static_cast<const typename Side::type *>(a.side) + row * a.side_stride + first;
  typename Side::type *side_out = kMode == kResidual ? static_cast<typename Side::type *>(a.side_out) + row * a.width + first : nullptr;
  const float *w = a.weight + first;

  const int pieces = (a.n + kPiece - 1) / kPiece;
  constexpr int kKeep = kHold > 0 ? kHold : 1;
  float v[kKeep][kPiece], g[kMode == kNormFirst ? kKeep : 1][kPiece];
  float sums[kKeep] = {};
  auto fetch = [&](int p, float x[kPiece], float s[kPiece]) {
    const int at = p * kPiece, left = a.n - at;
    Io::load(in + at, left, x);
    if (side != nullptr) {
      Side::load(side + at, left, s);
    } else {
#pragma unroll
      for (int i = 0; i < kPiece; ++i) s[i] = 0.f;
    }
  };
  if (kHold > 0) {
    float s[kKeep][kPiece];
#pragma unroll
    for (int k = 0; k < kKeep; ++k)
      if (t + k * kThreads < pieces) fetch(t + k * kThreads, v[k], s[k]);
#pragma unroll
    for (int k = 0; k < kKeep; ++k)
      if (t + k * kThreads < pieces) {
        combine<kMode>(v[k], s[k], a.scale);
#pragma unroll
        for (int i = 0; i < kPiece; ++i) {
          sums[k] = fmaf(v[k][i], v[k][i], sums[k]);
          if (kMode == kNormFirst) g[k][i] = s[k][i];
        }
      }
  } else {
    for (int p = t; p < pieces; p += kThreads) {
      float s[kPiece];
      fetch(p, v[0], s);
      combine<kMode>(v[0], s, a.scale);
#pragma unroll
      for (int i = 0; i < kPiece; ++i) sums[0] = fmaf(v[0][i], v[0][i], sums[0]);
    }
  }
#pragma unroll
  for (int k = 0; k < kKeep; ++k)
#pragma unroll
    for (int d = (kThreads < 64 ? kThreads : 64) / 2; d > 0; d >>= 1) sums[k] += __shfl_xor(sums[k], d);
  float sum = sums[0];
  if (kWaves > 1) {
    __shared__ float part[kKeep * kWaves];
    if ((threadIdx.x & 63) == 0)
#pragma unroll
      for (int k = 0; k < kKeep; ++k) part[k * kWaves + threadIdx.x / 64] = sums[k];
    __syncthreads();
    sum = part[0];
#pragma unroll
    for (int i = 1; i < kKeep * kWaves; ++i) sum += part[i];
  }
  const float r = 1.f / sqrtf(fmaf(sum, a.inv_n, a.eps));
  auto finish = [&](int p, const float x[kPiece], const float *gate) {
    const int at = p * kPiece, left = a.n - at;
    float wv[kPiece], o[kPiece];
    F32::load(w + at, left, wv);
#pragma unroll
    for (int i = 0; i < kPiece; ++i) o[i] = x[i] * r * wv[i] * (kMode == kNormFirst ? gate[i] : 1.f);
    Io::store(out + at, left, o);
    if (kMode == kResidual) Side::store(side_out + at, left, x);
  };
  if (kHold > 0) {
#pragma unroll
    for (int k = 0; k < kKeep; ++k)
      if (t + k * kThreads < pieces) finish(t + k * kThreads, v[k], g[kMode == kNormFirst ? k : 0]);
  } else {
    // (a thread reads again what it read before, and writes there only: outputs that are inputs are no hazard)
    for (int p = t; p < pieces; p += kThreads) {
      float s[kPiece];
      fetch(p, v[0], s);
      combine<kMode>(v[0], s, a.scale);
      finish(p, v[0], s);
    }
  }
}

template <typename Io, typename Side, int kMode, int kThreads, int kHold>
hipError_t launch_shape(NormArgs a, hipStream_t stream) {
  constexpr int kBlock = kThreads < 256 ? 256 : kThreads, kUnits = kBlock / kThreads;
  constexpr int64_t kMost = kMostThreads / kBlock * kUnits;
  hipError_t e = hipSuccess;
  for (; a.first < a.units && e == hipSuccess; a.first += kMost) {
    const int64_t units = std::min(a.units - a.first, kMost);
    hipLaunchKernelGGL((norm_kernel<Io, Side, kMode, kThreads, kHold>), dim3(static_cast<unsigned>((units + kUnits - 1) / kUnits)), dim3(kBlock), 0,
                       stream, a);
    e = hipGetLastError();
  }
  return e;
}

// Threads and pieces a thread by the unit's width: no more registers than the pieces need, which leave room for other units'
// requests (16384 rows of 5120 bf16 values: 132 us with four pieces a thread, of which two and a half are there, 100 with three),
// and no wave with nothing to do.  Few units leave CUs idle, and each is a chain of latencies: a piece a thread, where that is
// possible (5120 bf16 values: one row 3.1 us instead of 4.2, 512 rows 5.5 and 6.7, 1024 rows 8.5 and 8.4).
template <typename Io, typename Side, int kMode>
hipError_t launch_mode(const NormArgs &a, hipStream_t stream) {
  const int pieces = (a.n + kPiece - 1) / kPiece;
  if (pieces <= 16) return launch_shape<Io, Side, kMode, 16, 1>(a, stream);
  if (pieces <= 64) return launch_shape<Io, Side, kMode, 64, 1>(a, stream);
  if (pieces <= 256) return launch_shape<Io, Side, kMode, 256, 1>(a, stream);
  if (a.units <= kFewUnits && pieces <= 2048) {
    if (pieces <= 512) return launch_shape<Io, Side, kMode, 512, 1>(a, stream);
    if (pieces <= 1024) return launch_shape<Io, Side, kMode, 1024, 1>(a, stream);
    return launch_shape<Io, Side, kMode, 1024, 2>(a, stream);
  }
  if (pieces <= 512) return launch_shape<Io, Side, kMode, 256, 2>(a, stream);
  if (pieces <= 768) return launch_shape<Io, Side, kMode, 256, 3>(a, stream);
  if (pieces <= 1024) return launch_shape<Io, Side, kMode, 512, 2>(a, stream);
  if (pieces <= 2048) return launch_shape<Io, Side, kMode, 512, 4>(a, stream);
  return launch_shape<Io, Side, kMode, 1024, 0>(a, stream);
}

}  // namespace

hipError_t launch_norm_gated(int64_t rows, int width, int groups, bool bf16, const void *y, const void *z, int64_t z_stride,
                             const float *weight, float eps, bool norm_first, void *out, hipStream_t stream) {
  NormArgs a = {};
  a.in = y;
  a.side = z;
  a.weight = weight;
  a.out = out;
  a.units = rows * groups;
  a.side_stride = z_stride;
  a.width = width;
  a.n = width / groups;
  a.groups = groups;
  a.eps = eps;
  a.inv_n = 1.f / static_cast<float>(a.n);
  if (bf16) return norm_first ? launch_mode<Bf16, Bf16, kNormFirst>(a, stream) : launch_mode<Bf16, Bf16, kGateFirst>(a, stream);
  return norm_first ? launch_mode<F32, F32, kNormFirst>(a, stream) : launch_mode<F32, F32, kGateFirst>(a, stream);
}

hipError_t launch_norm_residual(int64_t rows, int width, bool bf16, bool stream_bf16, const void *x, const void *residual,
                                float scale, const float *weight, float eps, void *out, void *residual_out, hipStream_t stream) {
  NormArgs a = {};
  a.in = x;
  a.side = residual;
  a.weight = weight;
  a.out = out;
  a.side_out = residual_out;
  a.units = rows;
  a.side_stride = width;
  a.width = width;
  a.n = width;
  a.groups = 1;
  a.scale = scale;
  a.eps = eps;
  a.inv_n = 1.f / static_cast<float>(width);
  if (!bf16) return launch_mode<F32, F32, kResidual>(a, stream);
  return stream_bf16 ? launch_mode<Bf16, Bf16, kResidual>(a, stream) : launch_mode<Bf16, F32, kResidual>(a, stream);
}

}  // namespace ssd
