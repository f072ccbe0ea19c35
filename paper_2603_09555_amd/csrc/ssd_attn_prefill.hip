// Causal attention of packed new tokens over a paged cache:  y[t][h] = sum_s softmax_s(scale q[t][h] . K[s]) V[s], s up to t's
// position.
//
// Bound by the matrix pipe for prompts, by the pass over K and V for a few new tokens behind a long cache.  The rows of a unit
// are 128 (token, head) pairs of one sequence and key head, tokens slowest, so that a key head's query heads share its K and V;
// a wave has 32 of them as the columns of 32 x 32 matrix products and keeps their running maximum m, sum l and O^T in registers:
//
//   S^T (tokens x rows) = K Q^T,   p = 2^(S - m),   O^T (values x rows) += V^T P^T
//
// Tiles of K and V (64 tokens; fp32: 32) go through LDS, the next one being on its way while one is worked on.  The first
// product leaves a lane with tokens 8i + 4h .. 8i + 4h + 3 (h = lane / 32) of its row; these are what it supplies as the second
// operand of V^T P^T, whose first operand comes from LDS with the same order of tokens (bf16: by transposing reads).
//
// Where there are few units, several workgroups share one's tokens and leave (m, l, O) in the workspace for a second launch.
#include "ssd_attn.hpp"

namespace ssd {
namespace {

using namespace block;

constexpr int kWaves = 4, kThreads = 64 * kWaves, kWaveRows = 32, kUnitRows = kWaves * kWaveRows;
constexpr int kSplitTiles = 8;     // tiles a workgroup has at least when a unit is shared
constexpr int kWantedUnits = 512;  // workgroups that fill the GPU
constexpr float kNone = -3.0e38f;  // a maximum of nothing: finite, so that differences are numbers
// The running maximum follows a larger one only when that is 2^kSlack times more: until then probabilities are up to 2^kSlack,
// which costs no accuracy, and O need not be scaled again.
constexpr float kSlack = 8.f;

struct PrefillArgs {
  const int32_t *cu, *lens, *table;
  const void *q, *k, *v;
  void *y;
  float *part;       // per unit and split: kUnitRows x (D + 4): O, m, l
  AttnDims d;
  uint32_t inv_group;
  int units;         // at most, of a key head
  int splits;        // at most, of a unit
  float scale_log2;  // scale * log2(e)
};

// A unit's rows and the tokens they see.
struct Unit {
  int rows;        // 0: there is no such unit
  int first_row;   // of its sequence
  int seq, begin;  // the sequence and its first new token
  int pos0;        // that token's position
  int base, tiles, splits;
};
template <int kTokens>
__device__ __forceinline__ Unit find_unit(const PrefillArgs &a, int u) {
  Unit r = {};
  // Sequence b's units begin at cu[b] * group / rows + b: these are at least as far apart as its units are many.
  const auto bound = [&](int b) { return min(max(a.cu[b], 0), a.d.T); };
  const auto first_unit = [&](int b) { return static_cast<int64_t>(bound(b)) * a.d.G / kUnitRows + b; };
  int last = -1;
  for (int b0 = 0; b0 < a.d.B; b0 += 64) {
    const int b = b0 + (threadIdx.x & 63);
    const uint64_t m = __ballot(b < a.d.B && first_unit(b) <= u);
    if (m != 0) last = b0 + 63 - __builtin_clzll(m);
  }
  if (last < 0) return r;
  r.seq = last;
  r.begin = bound(last);
  const int count = bound(last + 1) - r.begin;
  const int64_t first = (u - first_unit(last)) * kUnitRows, all = static_cast<int64_t>(count) * a.d.G;
  if (first >= all) return r;
  r.first_row = static_cast<int>(first);
  r.rows = static_cast<int>(min(static_cast<int64_t>(kUnitRows), all - first));
  const int len = cut_length(a.d, a.lens[last]);
  r.pos0 = len - count;
  const int lowest = r.pos0 + quotient(r.first_row, a.d.G, a.inv_group);
  const int highest = r.pos0 + quotient(r.first_row + r.rows - 1, a.d.G, a.inv_group);
  r.base = (a.d.window > 0 ? max(0, lowest + 1 - a.d.window) : 0) & ~(kTokens - 1);
  r.tiles = highest < 0 ? 0 : (highest + 1 - r.base + kTokens - 1) / kTokens;
  r.splits = max(1, min(a.splits, r.tiles / kSplitTiles));
  return r;
}

__device__ __forceinline__ f32x16 mfma_bf16(u32x4 a, u32x4 b, f32x16 c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}
__device__ __forceinline__ f32x16 mfma_f32(float a, float b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x2f32(a, b, c, 0, 0, 0); }

// Transposed LDS read (ds_read_b64_tr_b16): in each group of 16 lanes, lane i names four neighbouring 16-bit values, of row i / 4
// and columns 4 (i % 4) on, and receives column i of the four rows.
__device__ __forceinline__ u32x2 lds_transposed(const char *p) {
  typedef short s16x4 __attribute__((ext_vector_type(4)));
  typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
  return __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)(uint32_t)(uintptr_t)p));
}

// Geometry of a tile in LDS for head vectors of up to DP values (D are there, the others are zeros): rows of kPieces pieces of 16
// bytes, in an order that depends on the row so that the reads of either product go to all banks.
template <bool kBf16, int DP>
struct Geometry {
  static constexpr int kSize = kBf16 ? 2 : 4;
  static constexpr int kTokens = kBf16 ? 64 : 32;
  static constexpr int kRowBytes = DP * kSize, kPieces = kRowBytes / 16;
  static constexpr int kTileBytes = kTokens * kRowBytes;
  static constexpr int kFetch = kTokens * kPieces / kThreads;  // pieces of a tile a thread brings
  // 16 lanes read the same piece of neighbouring rows
  static __device__ __forceinline__ int key_piece(int row, int c) { return c ^ (row & (kPieces < 16 ? kPieces - 1 : 15)); }
  // bf16: 32 lanes read 64 bytes of four neighbouring rows; fp32: 128 of one
  static __device__ __forceinline__ int value_piece(int row, int c) {
    return !kBf16 ? c : DP == 64 ? c ^ ((row & 2) << 1) : c ^ ((row & 3) << 2);
  }
};

template <bool kBf16, int DP>
__global__ __launch_bounds__(kThreads, DP == 256 ? 1 : 2) void prefill_kernel(const PrefillArgs a) {
  using Geo = Geometry<kBf16, DP>;
  constexpr int kTokens = Geo::kTokens, kHalves = kTokens / 32, kColTiles = DP / 32;
  constexpr int kQueryPieces = DP * Geo::kSize / 32;  // of 16 bytes, a lane
  __shared__ char lds[2][2][Geo::kTileBytes];         // two tiles of K and V

  int id = blockIdx.x;
  const int split = id % a.splits;
  id /= a.splits;
  const int hk = id % a.d.Hk;
  const Unit unit = find_unit<kTokens>(a, a.units - 1 - id / a.d.Hk);  // (the last units see the most tokens)
  if (unit.rows == 0 || split >= unit.splits) return;

  const int lane = threadIdx.x & 63, wave = threadIdx.x / 64, n = lane & 31, h = lane / 32;
  const int bytes = a.d.D * Geo::kSize;
  const int64_t page_bytes = (static_cast<int64_t>(a.d.Hk) << a.d.lg_page) * bytes;
  const int page_mask = (1 << a.d.lg_page) - 1;
  const char *kh = static_cast<const char *>(a.k) + (static_cast<int64_t>(hk) << a.d.lg_page) * bytes;
  const char *vh = static_cast<const char *>(a.v) + (static_cast<int64_t>(hk) << a.d.lg_page) * bytes;
  const int32_t *table = a.table + static_cast<int64_t>(unit.seq) * a.d.max_pages;

  // this lane's row
  const int local = wave * kWaveRows + n;
  const bool mine = local < unit.rows;
  const int row = unit.first_row + min(local, unit.rows - 1), token = quotient(row, a.d.G, a.inv_group);
  const int pos = unit.pos0 + token;
  const int64_t out_row = static_cast<int64_t>(unit.begin + token) * a.d.H + hk * a.d.G + (row - token * a.d.G);
  const int seen_from = a.d.window > 0 ? pos - a.d.window + 1 : 0;  // (a position)
  // of the wave: every row sees [all_from, all_to], none sees beyond any_to
  const int all_to = __builtin_amdgcn_readfirstlane(pos), any_to = __builtin_amdgcn_readlane(pos, 31);
  const int all_from = __builtin_amdgcn_readlane(seen_from, 31);
  const bool idle = wave * kWaveRows >= unit.rows;

  u32x4 query[kQueryPieces];
#pragma unroll
  for (int i = 0; i < kQueryPieces; ++i) {
    const int byte = 32 * i + 16 * h;
    query[i] = u32x4{0u, 0u, 0u, 0u};
    if (mine && byte < bytes) query[i] = *reinterpret_cast<const u32x4 *>(static_cast<const char *>(a.q) + out_row * bytes + byte);
  }
  f32x16 o[kColTiles];
#pragma unroll
  for (int c = 0; c < kColTiles; ++c)
#pragma unroll
    for (int r = 0; r < 16; ++r) o[c][r] = 0.f;
  float m = kNone, l = 0.f;

  const int tile0 = static_cast<int>(static_cast<int64_t>(unit.tiles) * split / unit.splits);
  const int tile1 = static_cast<int>(static_cast<int64_t>(unit.tiles) * (split + 1) / unit.splits);
  const int end = unit.pos0 + quotient(unit.first_row + unit.rows - 1, a.d.G, a.inv_group) + 1;  // tokens seen by any row

  u32x4 fetched[2][Geo::kFetch];
  uint64_t gone = 0, gone_next = 0;  // tokens of the tile whose page is not in the cache
  auto fetch = [&](int tile) {
    const int first = unit.base + tile * kTokens;
    const int t = min(first + (lane & (kTokens - 1)), end - 1);
    int page = table[t >> a.d.lg_page];
    const bool bad = static_cast<unsigned>(page) >= static_cast<unsigned>(a.d.npages);
    gone_next = __ballot(bad) & (kTokens == 64 ? ~0ull : (1ull << kTokens) - 1);
    if (bad) page = -1;
#pragma unroll
    for (int i = 0; i < Geo::kFetch; ++i) {
      const int piece = threadIdx.x + i * kThreads, r = piece / Geo::kPieces, c = piece % Geo::kPieces;
      const int where = __shfl(page, r);
      const int at = min(first + r, end - 1) & page_mask;
      fetched[0][i] = fetched[1][i] = u32x4{0u, 0u, 0u, 0u};
      // (a token behind the last one that is seen is brought as zeros: its probability is zero, and so must be the product)
      if (where >= 0 && 16 * c < bytes && first + r < end) {
        const int64_t byte = where * page_bytes + static_cast<int64_t>(at) * bytes + 16 * c;
        fetched[0][i] = *reinterpret_cast<const u32x4 *>(kh + byte);
        fetched[1][i] = *reinterpret_cast<const u32x4 *>(vh + byte);
      }
    }
  };
  auto stage = [&](int buffer) {
#pragma unroll
    for (int i = 0; i < Geo::kFetch; ++i) {
      const int piece = threadIdx.x + i * kThreads, r = piece / Geo::kPieces, c = piece % Geo::kPieces;
      *reinterpret_cast<u32x4 *>(&lds[buffer][0][r * Geo::kRowBytes + 16 * Geo::key_piece(r, c)]) = fetched[0][i];
      *reinterpret_cast<u32x4 *>(&lds[buffer][1][r * Geo::kRowBytes + 16 * Geo::value_piece(r, c)]) = fetched[1][i];
    }
    gone = gone_next;
  };

  if (tile0 < tile1) {
    fetch(tile0);
    stage(0);
  }
  __syncthreads();
  for (int tile = tile0; tile < tile1; ++tile) {
    const int buffer = (tile - tile0) & 1, first = unit.base + tile * kTokens;
    const char *kt = lds[buffer][0], *vt = lds[buffer][1];
    const uint64_t gone_now = gone;
    if (tile + 1 < tile1) fetch(tile + 1);
    if (!idle && first <= any_to) {
      f32x16 s[kHalves];
#pragma unroll
      for (int t = 0; t < kHalves; ++t) {
#pragma unroll
        for (int r = 0; r < 16; ++r) s[t][r] = 0.f;
        const char *krow = kt + (32 * t + n) * Geo::kRowBytes;
#pragma unroll
        for (int i = 0; i < kQueryPieces; ++i) {
          const u32x4 k = *reinterpret_cast<const u32x4 *>(krow + 16 * Geo::key_piece(n, 2 * i + h));
          if constexpr (kBf16) {
            s[t] = mfma_bf16(k, query[i], s[t]);
          } else {
#pragma unroll
            for (int e = 0; e < 4; ++e) s[t] = mfma_f32(__uint_as_float(k[e]), __uint_as_float(query[i][e]), s[t]);
          }
        }
      }
      if (first + kTokens - 1 > all_to || first < all_from || gone_now != 0) {
#pragma unroll
        for (int t = 0; t < kHalves; ++t)
#pragma unroll
          for (int r = 0; r < 16; ++r) {
            const int in_tile = 32 * t + 8 * (r / 4) + 4 * h + r % 4, at = first + in_tile;
            if (at > pos || at < seen_from || ((gone_now >> in_tile) & 1)) s[t][r] = -INFINITY;
          }
      }
      float top = s[0][0];
#pragma unroll
      for (int t = 0; t < kHalves; ++t)
#pragma unroll
        for (int r = 0; r < 16; ++r) top = fmaxf(top, s[t][r]);
      top = fmaxf(top, __shfl_xor(top, 32)) * a.scale_log2;
      if (__any(top > m + kSlack)) {
        const float next = fmaxf(m, top), keep = __builtin_amdgcn_exp2f(m - next);
        m = next;
        l *= keep;
#pragma unroll
        for (int c = 0; c < kColTiles; ++c)
#pragma unroll
          for (int r = 0; r < 16; ++r) o[c][r] *= keep;
      }
#pragma unroll
      for (int t = 0; t < kHalves; ++t)
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          s[t][r] = __builtin_amdgcn_exp2f(fmaf(s[t][r], a.scale_log2, -m));
          l += s[t][r];
        }
      if constexpr (kBf16) {
        const char *vlane = vt + (4 * h + (lane & 15) / 4) * Geo::kRowBytes;
        const int byte = 32 * ((lane >> 4) & 1) + 8 * (lane & 3), vrow = (lane & 15) / 4;  // (4 h and multiples of 8 rows leave row & 3)
#pragma unroll
        for (int g = 0; g < 2 * kHalves; ++g) {  // 16 tokens
          u32x4 p;
#pragma unroll
          for (int i = 0; i < 4; ++i) p[i] = pack2(s[g / 2][8 * (g % 2) + 2 * i], s[g / 2][8 * (g % 2) + 2 * i + 1]);
#pragma unroll
          for (int c = 0; c < kColTiles; ++c) {
            const int piece = Geo::value_piece(vrow, 4 * c + byte / 16);
            const u32x2 lo = lds_transposed(vlane + 16 * g * Geo::kRowBytes + 16 * piece + byte % 16);
            const u32x2 hi = lds_transposed(vlane + (16 * g + 8) * Geo::kRowBytes + 16 * piece + byte % 16);
            o[c] = mfma_bf16(u32x4{lo[0], lo[1], hi[0], hi[1]}, p, o[c]);
          }
        }
      } else {
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          const float *vrow = reinterpret_cast<const float *>(vt + (8 * (r / 4) + 4 * h + r % 4) * Geo::kRowBytes);
#pragma unroll
          for (int c = 0; c < kColTiles; ++c) o[c] = mfma_f32(vrow[32 * c + n], s[0][r], o[c]);
        }
      }
    }
    if (tile + 1 < tile1) stage(buffer ^ 1);
    __syncthreads();
  }

  l += __shfl_xor(l, 32);
  if (!mine) return;
  if (unit.splits == 1) {
    const float inv = l == 0.f ? 0.f : 1.f / l;
#pragma unroll
    for (int c = 0; c < kColTiles; ++c)
#pragma unroll
      for (int r = 0; r < 16; r += 4) {
        const int col = 32 * c + 2 * r + 4 * h;
        if (col >= a.d.D) continue;
        if constexpr (kBf16) {
          const u32x2 q = {pack2(o[c][r] * inv, o[c][r + 1] * inv), pack2(o[c][r + 2] * inv, o[c][r + 3] * inv)};
          *reinterpret_cast<u32x2 *>(static_cast<uint16_t *>(a.y) + out_row * a.d.D + col) = q;
        } else {
          const f32x4 q = {o[c][r] * inv, o[c][r + 1] * inv, o[c][r + 2] * inv, o[c][r + 3] * inv};
          *reinterpret_cast<f32x4 *>(static_cast<float *>(a.y) + out_row * a.d.D + col) = q;
        }
      }
  } else {
    float *part = a.part + (static_cast<int64_t>(blockIdx.x) * kUnitRows + local) * (a.d.D + 4);
#pragma unroll
    for (int c = 0; c < kColTiles; ++c)
#pragma unroll
      for (int r = 0; r < 16; r += 4) {
        const int col = 32 * c + 2 * r + 4 * h;
        if (col < a.d.D) *reinterpret_cast<f32x4 *>(part + col) = f32x4{o[c][r], o[c][r + 1], o[c][r + 2], o[c][r + 3]};
      }
    if (h == 0) {
      part[a.d.D] = m;
      part[a.d.D + 1] = l;
    }
  }
}

// Joins the splits of a unit: one workgroup for kJoinRows of its rows.
constexpr int kJoinRows = 16;
template <bool kBf16>
__global__ __launch_bounds__(kThreads) void prefill_join_kernel(const PrefillArgs a) {
  int id = blockIdx.x;
  const int cut = id % (kUnitRows / kJoinRows);
  id /= kUnitRows / kJoinRows;
  const int hk = id % a.d.Hk;
  const Unit unit = find_unit<kBf16 ? 64 : 32>(a, a.units - 1 - id / a.d.Hk);
  if (unit.rows <= cut * kJoinRows || unit.splits == 1) return;
  const int cols = a.d.D / 4;
  for (int e = threadIdx.x; e < kJoinRows * cols; e += kThreads) {
    const int local = cut * kJoinRows + e / cols, col = 4 * (e % cols);
    if (local >= unit.rows) break;
    const float *part = a.part + (static_cast<int64_t>(id) * a.splits * kUnitRows + local) * (a.d.D + 4);
    const int64_t step = static_cast<int64_t>(kUnitRows) * (a.d.D + 4);
    float top = kNone, sum = 0.f;
    f32x4 v = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
    for (int s = 0; s < unit.splits; ++s, part += step) {
      const float m = part[a.d.D], l = part[a.d.D + 1];
      const f32x4 o = *reinterpret_cast<const f32x4 *>(part + col);
      const float next = fmaxf(top, m), keep = __builtin_amdgcn_exp2f(top - next), f = __builtin_amdgcn_exp2f(m - next);
      top = next;
      sum = fmaf(sum, keep, l * f);
#pragma unroll
      for (int r = 0; r < 4; ++r) v[r] = fmaf(v[r], keep, o[r] * f);
    }
    const float inv = sum == 0.f ? 0.f : 1.f / sum;
    const int row = unit.first_row + local, token = quotient(row, a.d.G, a.inv_group);
    const int64_t at = (static_cast<int64_t>(unit.begin + token) * a.d.H + hk * a.d.G + (row - token * a.d.G)) * a.d.D + col;
    if constexpr (kBf16) {
      const u32x2 q = {pack2(v[0] * inv, v[1] * inv), pack2(v[2] * inv, v[3] * inv)};
      *reinterpret_cast<u32x2 *>(static_cast<uint16_t *>(a.y) + at) = q;
    } else {
      *reinterpret_cast<f32x4 *>(static_cast<float *>(a.y) + at) = f32x4{v[0] * inv, v[1] * inv, v[2] * inv, v[3] * inv};
    }
  }
}

struct Plan {
  int units, splits;
};
Plan plan_of(const AttnDims &d) {
  Plan p;
  p.units = static_cast<int>(static_cast<int64_t>(d.T) * d.G / kUnitRows + d.B);
  const int64_t all = static_cast<int64_t>(p.units) * d.Hk;
  const int64_t tiles = d.capacity() / (d.bf16 ? 64 : 32);
  const int64_t wanted = (kWantedUnits + all - 1) / all, most = tiles / kSplitTiles;
  p.splits = static_cast<int>(wanted < most ? wanted : most);
  if (p.splits < 1) p.splits = 1;
  return p;
}

template <bool kBf16>
hipError_t launch(const PrefillArgs &a, hipStream_t stream) {
  const dim3 grid(static_cast<unsigned>(a.units) * a.d.Hk * a.splits), threads(kThreads);
  if (a.d.D <= 64)
    hipLaunchKernelGGL((prefill_kernel<kBf16, 64>), grid, threads, 0, stream, a);
  else if (a.d.D <= 128)
    hipLaunchKernelGGL((prefill_kernel<kBf16, 128>), grid, threads, 0, stream, a);
  else
    hipLaunchKernelGGL((prefill_kernel<kBf16, 256>), grid, threads, 0, stream, a);
  if (const hipError_t e = hipGetLastError(); e != hipSuccess || a.splits == 1) return e;
  hipLaunchKernelGGL(prefill_join_kernel<kBf16>, dim3(static_cast<unsigned>(a.units) * a.d.Hk * (kUnitRows / kJoinRows)), threads, 0, stream, a);
  return hipGetLastError();
}

}  // namespace

size_t attn_prefill_workspace_bytes(const AttnDims &d) {
  const Plan p = plan_of(d);
  if (p.splits == 1) return 256;
  return (static_cast<size_t>(p.units) * d.Hk * p.splits * kUnitRows * (d.D + 4) * 4 + 255) / 256 * 256;
}

hipError_t launch_attn_prefill(const AttnDims &d, const int32_t *cu, const int32_t *lens, const int32_t *table, const void *q,
                               const void *k_cache, const void *v_cache, float scale, void *y, void *workspace,
                               hipStream_t stream) {
  const Plan p = plan_of(d);
  PrefillArgs a = {};
  a.cu = cu;
  a.lens = lens;
  a.table = table;
  a.q = q;
  a.k = k_cache;
  a.v = v_cache;
  a.y = y;
  a.part = static_cast<float *>(workspace);
  a.d = d;
  a.inv_group = inverse_of(d.G);
  a.units = p.units;
  a.splits = p.splits;
  a.scale_log2 = scale * 1.44269504f;
  return d.bf16 ? launch<true>(a, stream) : launch<false>(a, stream);
}

}  // namespace ssd
