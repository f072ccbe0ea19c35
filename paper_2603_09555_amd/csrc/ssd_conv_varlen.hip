// Depthwise causal convolution of a packed batch of prompts of any lengths (or of later pieces of prompts):
//
//   z[t][c]  = act( bias[c] + sum_j w[c][j] * window_t[j][c] ),  window_t = the k-1 inputs before token t of its sequence, u_t
//   cache[q] <- the last k-1 inputs of sequence q                          (channels, k-1)
//
// Inputs before a sequence's first token come from its cache, or are zero.  Bound by one read of u and one write of z, or by
// latency where there are few tokens.  A thread owns one channel of fp32 or two of bf16 (one where an output's width is odd), 4 bytes
// either way, and a run of the packed tokens, whatever sequences these belong to, with the window and its weights in registers.  It
// finds the sequence of its first token once, while its first rows are on their way; where the next one begins it fills the window
// from that one's cache.  Rows of u may be a slice of wider ones, so that the input projection's output need not be copied.
//
// 18929 tokens of 12 prompts, 5376 channels, bf16: 86.7 us, 4.7 TB/s; 4886 x 1536 in fp32 12.2 us, 4.9 TB/s; 13 x 1792 4.4 us.  Beside
// each other: 4, 8 and 16 bytes a lane 88, 91 and 92 us (97 with loads that leave the caches alone), fp32 13.9, 14.7 and 14.5.
//
// The caches are left by threads of their own, one a sequence and channel: in the same launch, or, where they are updated in
// place, in one behind it (a sequence's first run reads what its last would write), which takes 3.3 us: 13 x 1792 7.4 us in place and
// 4.1 out of place, 18929 x 5376 89.8 and 86.5.
#include <algorithm>

#include "ssd_conv.hpp"

namespace ssd {
namespace {

// Tokens a thread, at least: few tokens are worth more threads, and a launch takes 2^32.
constexpr int64_t kMostThreads = int64_t{1} << 31;
int shortest_run(int T, int64_t groups) { return static_cast<int>(std::max<int64_t>(4, (T * groups + kMostThreads - 1) / kMostThreads)); }

struct VarlenArgs {
  const void *u;
  int64_t u_stride;
  const float *w, *bias;
  const int32_t *cu;
  const void *state_in;
  void *state_out;
  ConvOut out;
  int B, T, C, act;
  int run;                   // tokens a thread
  unsigned filter_blocks;    // workgroups in front of those that leave the caches
};

// V neighbouring channels of a row; addresses need no more than the element's alignment.
template <typename Io, int V>
struct Row {
  typename Io::type e[V];
};
template <typename Io, int V>
__device__ __forceinline__ Row<Io, V> load_row(const typename Io::type *p) {
  Row<Io, V> r;
  if constexpr (V == 1) {
    r.e[0] = *p;
  } else {
    static_assert(V == 2 && sizeof(r) == 4, "one channel, or two of bf16");
    typedef uint32_t __attribute__((aligned(2))) Pair;
    const uint32_t q = *reinterpret_cast<const Pair *>(p);
    __builtin_memcpy(&r, &q, sizeof(r));
  }
  return r;
}
template <typename Io>
__device__ __forceinline__ float to_float(typename Io::type v) {
  return Io::load(&v, 0);
}

// A thread looks several boundaries up, one after another: they go through LDS where they fit.  Which it is has to be known to the
// compiler: through a pointer to either it makes flat loads, which choose the memory by the address in front of the constant that
// they add, and fault where that address is not in LDS while the sum is.
constexpr int kMostStaged = 1024;

template <typename Io, int K>
__device__ __forceinline__ void leave_cache(const VarlenArgs &a, int64_t i) {
  using E = typename Io::type;
  const int q = static_cast<int>(i / a.C), c = static_cast<int>(i - static_cast<int64_t>(q) * a.C);
  const int begin = max(a.cu[q], 0), len = max(min(a.cu[q + 1], a.T) - begin, 0);
  const E *const before = static_cast<const E *>(a.state_in) + (a.state_in ? i * (K - 1) : 0);
  const E *const u = static_cast<const E *>(a.u) + static_cast<int64_t>(begin) * a.u_stride + c;
  E keep[K - 1];
#pragma unroll
  for (int j = 0; j + 1 < K; ++j) {
    const int t = len - (K - 1) + j;  // of the sequence's new tokens; negative: cached before
    if (t >= 0) keep[j] = u[t * a.u_stride];
    else keep[j] = a.state_in ? before[K - 1 + t] : E(0);
  }
  E *const out = static_cast<E *>(a.state_out) + i * (K - 1);
#pragma unroll
  for (int j = 0; j + 1 < K; ++j) out[j] = keep[j];
}

template <typename Io, int K>
__global__ __launch_bounds__(kConvThreads) void conv_cache_kernel(const VarlenArgs a) {
  const int64_t i = static_cast<int64_t>(blockIdx.x) * kConvThreads + threadIdx.x;
  if (i < static_cast<int64_t>(a.B) * a.C) leave_cache<Io, K>(a, i);
}

template <typename Io, int V, int K, bool kStaged>
__global__ __launch_bounds__(kConvThreads) void conv_varlen_kernel(const VarlenArgs a) {
  using E = typename Io::type;
  if (blockIdx.x >= a.filter_blocks) {
    const int64_t i = static_cast<int64_t>(blockIdx.x - a.filter_blocks) * kConvThreads + threadIdx.x;
    if (i < static_cast<int64_t>(a.B) * a.C) leave_cache<Io, K>(a, i);
    return;
  }
  __shared__ int32_t staged[kStaged ? kMostStaged + 1 : 1];  // [q + 1]: boundary q
  if constexpr (kStaged) {
    for (int i = threadIdx.x; i <= a.B; i += kConvThreads) staged[i + 1] = a.cu[i];
    __syncthreads();
  }
  auto cu = [&](int q) __attribute__((always_inline)) {
    if constexpr (kStaged) return staged[q + 1];
    else return a.cu[q];
  };
  const unsigned groups = a.C / V, gid = blockIdx.x * kConvThreads + threadIdx.x;
  const unsigned run = gid / groups;
  const int64_t first = static_cast<int64_t>(run) * a.run;
  if (first >= a.T) return;
  const int t0 = static_cast<int>(first), t1 = min(a.T, t0 + a.run);
  const int c0 = static_cast<int>(gid - run * groups) * V;
  const E *const u = static_cast<const E *>(a.u) + c0;
  const E *const cached = static_cast<const E *>(a.state_in) + (a.state_in ? static_cast<int64_t>(c0) * (K - 1) : 0);

  constexpr int kBatch = 4;
  struct Rows {
    Row<Io, V> r[kBatch];
  } buf[2];
  auto request = [&](Rows &r, int tb) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < kBatch; ++i) r.r[i] = load_row<Io, V>(u + min(tb + i, t1 - 1) * a.u_stride);  // (surplus ones: the last row)
  };
  // all that does not depend on the boundaries: the first rows, those in front of them (which may be another sequence's), weights
  Row<Io, V> front[K - 1];
#pragma unroll
  for (int j = 0; j + 1 < K; ++j) front[j] = load_row<Io, V>(u + max(t0 - (K - 1) + j, 0) * a.u_stride);
  request(buf[0], t0);
  float wt[V][K], bs[V];
#pragma unroll
  for (int v = 0; v < V; ++v)
#pragma unroll
    for (int j = 0; j < K; ++j) wt[v][j] = a.w[static_cast<int64_t>(c0 + v) * K + j];
#pragma unroll
  for (int v = 0; v < V; ++v) bs[v] = 0.f;
  if (a.bias) {
#pragma unroll
    for (int v = 0; v < V; ++v) bs[v] = a.bias[c0 + v];
  }
  // tokens [begin, end) are sequence next - 1's; those in front of the first and behind the last one are in none
  int next = 0, begin = 0, end = t0;
  for (int most = a.B; next < most;) {
    const int middle = (next + most) / 2;
    if (cu(middle) <= t0) next = middle + 1;
    else most = middle;
  }
  float win[K][V];
  // win[1 ..]: the inputs in front of a token that `behind` new ones of its sequence precede; `behind` of them are there already
  auto fill_cached = [&](int behind) __attribute__((always_inline)) {
#pragma unroll
    for (int j = 1; j < K; ++j)
      if (K - j > behind) {
#pragma unroll
        for (int v = 0; v < V; ++v)
          win[j][v] = a.state_in ? to_float<Io>(cached[(static_cast<int64_t>(next - 1) * a.C + v) * (K - 1) + j - 1 + behind]) : 0.f;
      }
  };
  // `turn`: the next token at which something changes; `inside`: whether the tokens up to it are in a sequence
  int turn;
  bool inside;
  auto enter = [&](int t) __attribute__((always_inline)) {
    while (next < a.B && cu(next) <= t) ++next;
    if (next > 0) {
      begin = max(cu(next - 1), 0);
      end = min(cu(next), a.T);
    }
    inside = next > 0 && t >= begin && t < end;
    turn = inside ? end : next < a.B ? max(cu(next), t + 1) : a.T;
  };
  enter(t0);
#pragma unroll
  for (int j = 1; j < K; ++j)
#pragma unroll
    for (int v = 0; v < V; ++v) win[j][v] = to_float<Io>(front[j - 1].e[v]);
  if (inside && t0 - begin < K - 1) fill_cached(t0 - begin);

  // (chosen without an index: the arguments are in scalar registers)
  const bool second = c0 >= a.out.begin[1], third = c0 >= a.out.begin[2];
  const int out_first = third ? a.out.begin[2] : second ? a.out.begin[1] : 0;
  const int width = (third ? a.out.begin[3] : second ? a.out.begin[2] : a.out.begin[1]) - out_first;
  E *const z = static_cast<E *>(third ? a.out.ptr[2] : second ? a.out.ptr[1] : a.out.ptr[0]) + (c0 - out_first);
  auto process = [&](const Rows &r, int tb) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < kBatch; ++i) {
      const int t = tb + i;
      if (t < t1) {
        if (t >= turn) {
          enter(t);
          if (inside) fill_cached(0);  // (a sequence's first token)
        }
#pragma unroll
        for (int j = 0; j + 1 < K; ++j)
#pragma unroll
          for (int v = 0; v < V; ++v) win[j][v] = win[j + 1][v];
#pragma unroll
        for (int v = 0; v < V; ++v) win[K - 1][v] = to_float<Io>(r.r[i].e[v]);
        float s[V];
#pragma unroll
        for (int v = 0; v < V; ++v) {
          s[v] = bs[v];
#pragma unroll
          for (int j = 0; j < K; ++j) s[v] = fmaf(wt[v][j], win[j][v], s[v]);
          s[v] = act_apply(s[v], a.act);
        }
        if (inside) {
          E *const zp = z + static_cast<int64_t>(t) * width;
          if constexpr (V == 1) Io::store(zp, 0, s[0]);
          else *reinterpret_cast<uint32_t *>(zp) = pack_bf16x2(s[0], s[1]);
        }
      }
    }
  };
  for (int tb = t0; tb < t1; tb += 2 * kBatch) {
    request(buf[1], tb + kBatch);
    process(buf[0], tb);
    request(buf[0], tb + 2 * kBatch);
    process(buf[1], tb + kBatch);
  }
}

template <typename Io, int V, int K>
int resident_blocks() {
  static const int blocks = [] {
    int n = 0;
    if (hipOccupancyMaxActiveBlocksPerMultiprocessor(&n, conv_varlen_kernel<Io, V, K, true>, kConvThreads, 0) != hipSuccess || n < 1) n = 4;
    return n;
  }();
  return blocks;
}

template <typename Io, int V, int K>
hipError_t varlen_launch(VarlenArgs a, hipStream_t stream) {
  const int groups = a.C / V;
  a.run = choose_run(a.T, groups, K, resident_blocks<Io, V, K>(), shortest_run(a.T, groups));
  const auto blocks = [](int64_t threads) { return static_cast<unsigned>((threads + kConvThreads - 1) / kConvThreads); };
  a.filter_blocks = blocks(static_cast<int64_t>((a.T + a.run - 1) / a.run) * groups);
  const unsigned cache_blocks = a.state_out ? blocks(static_cast<int64_t>(a.B) * a.C) : 0;
  const bool in_place = a.state_out != nullptr && a.state_out == a.state_in;
  const dim3 grid(a.filter_blocks + (in_place ? 0 : cache_blocks));
  if (a.B < kMostStaged)
    hipLaunchKernelGGL((conv_varlen_kernel<Io, V, K, true>), grid, dim3(kConvThreads), 0, stream, a);
  else
    hipLaunchKernelGGL((conv_varlen_kernel<Io, V, K, false>), grid, dim3(kConvThreads), 0, stream, a);
  if (const hipError_t e = hipGetLastError(); e != hipSuccess || !in_place) return e;
  hipLaunchKernelGGL((conv_cache_kernel<Io, K>), dim3(cache_blocks), dim3(kConvThreads), 0, stream, a);
  return hipGetLastError();
}
template <typename Io, int K>
hipError_t varlen_typed(const VarlenArgs &a, bool pairs, hipStream_t stream) {
  if constexpr (sizeof(typename Io::type) == 2) {
    if (pairs) return varlen_launch<Io, 2, K>(a, stream);
  }
  return varlen_launch<Io, 1, K>(a, stream);
}

}  // namespace

// Whether the threads of a call, one a channel and run, and one a channel and sequence, are no more than a launch takes.
bool conv_varlen_fits(int B, int T, int64_t C) { return shortest_run(T, C) <= kRunMax && B * C <= kMostThreads - 3 * kConvThreads; }

hipError_t launch_conv_varlen(int B, int T, int ksize, bool bf16, const int32_t *cu, const void *u, int64_t u_stride,
                              const float *w, const float *bias, const void *state_in, void *const z[3], const int width[3],
                              void *state_out, int act, hipStream_t stream) {
  VarlenArgs a = {};
  a.u = u;
  a.u_stride = u_stride;
  a.w = w;
  a.bias = bias;
  a.cu = cu;
  a.state_in = state_in;
  a.state_out = state_out;
  a.out = make_out(z, width);
  a.B = B;
  a.T = T;
  a.C = a.out.begin[3];
  a.act = act;
  const bool pairs = width[0] % 2 == 0 && width[1] % 2 == 0 && width[2] % 2 == 0;
  SSD_CONV_DISPATCH(varlen_typed, a, pairs, stream)
}

}  // namespace ssd
