// Attention of one new token of each sequence over a paged cache:  y[b][h] = sum_t softmax_t(scale q[b][h] . K[t]) V[t].
//
// Bound by the one pass over K and V.  The query heads of a key head (16 at a time) are the columns of 16 x 16 matrix products,
// so that K and V are read once for all of them:
//
//   S^T (tokens x heads) = K Q^T,   p = 2^(S - running maximum),   O^T (values x heads) = V^T P^T
//
// A wave walks tiles of 32 tokens by itself, with the running maximum m, sum l and O^T of its heads in registers, and no LDS:
//   * K's rows go from memory into the first operand as they lie (a lane holds 8 values of bf16, or 4 of fp32, of one token);
//   * the product leaves a lane with 8 of the 32 tokens of one head -- tokens 4j..4j+3 of either half, j = lane / 16 --, and a
//     contraction does not mind the order of its tokens: these eight are what the lane supplies as the second operand of V^T P^T;
//   * the first operand is then eight values of one column of V, from eight tokens.  A lane reads its eight tokens' rows, some
//     neighbouring columns of each, and makes the columns' operands by exchanging halves of registers (bf16; fp32 needs none).
//
// The waves of a workgroup take every kWaves-th tile of a unit (a sequence and key head) and are joined through LDS at its end.
// What hides the latency of memory is other waves' requests; where there are too few, the next tile's keys are asked for before
// this one is worked on, and its page numbers a tile earlier.
//
// Work is dealt by length: the visible tokens of all sequences and key heads, in blocks of 128, make one long list of which every
// workgroup takes an equal run, whatever the lengths are.  A unit within one workgroup is finished there; the others leave
// (m, l, O) in the workspace, which a second launch joins.  Where no sequence can be long, a workgroup of eight waves, or four
// where there are many units, takes a unit and there is no second launch.
//
// 32 heads over 8 of 128, bf16: 64 sequences to 32768 tokens 150 us, 5.9 TB/s of K and V; one of 32000 28 us, one of 518 8.8 us.
// fp32, 2 sequences to 100004, 10 heads over 2 of 64: 48 us, 4.2 TB/s, of which the joining launch is 5.
#include <algorithm>

#include "ssd_attn.hpp"

namespace ssd {
namespace {

using namespace block;

constexpr int kThreads = kDealers, kTile = 32, kBlock = kThreads / 64 * kTile, kRows = 16;
// Workgroups that work is dealt to: as many as are in work at a time, four to one a CU as their registers allow.
constexpr int workgroups_of(bool bf16, int dp) { return 256 * (dp == 256 ? 1 : bf16 ? (dp == 64 ? 4 : 3) : dp == 64 ? 3 : 2); }
constexpr int kMostWorkgroups = 1024;
constexpr unsigned kFewUnits = 256, kCUs = 256;
constexpr float kNone = -3.0e38f;  // a maximum of nothing: finite, so that differences are numbers
constexpr float kMost = 3.0e38f;   // the largest maximum: behind it, probabilities are infinite and y is not a number

// The workgroups that have blocks of a unit.  They write it down, so that the joining launch need not deal again.
struct Spread {
  int first, last;
};

struct StepArgs {
  const int32_t *lens, *table;
  const void *q, *k, *v;
  void *y;
  float *part;       // per workgroup two slots of kRows x (D + 2): O, m, l of a unit that began before its run, and of its last one
  Spread *spread;    // of each sequence's units
  AttnDims d;
  int row_tiles;     // of 16 heads, of a key head's heads
  int units;         // of a sequence
  int workgroups;    // that work is dealt to
  float scale_log2;  // scale * log2(e)
};

inline int row_tiles_of(const AttnDims &d) { return (d.G + kRows - 1) / kRows; }  // of 16 heads, of a key head's heads
inline int units_of(const AttnDims &d) { return d.Hk * row_tiles_of(d); }         // of a sequence

struct Span {
  int lo, len, base, blocks;  // tokens seen: [lo, len), in blocks of 128 from base on
};
__device__ __forceinline__ Span span_of(const StepArgs &a, int b) {
  Span s;
  s.len = max(a.lens[b], 0);
  if (s.len > a.d.capacity()) s.len = 0;  // (the new token has no place: it sees nothing)
  s.lo = a.d.window > 0 ? max(0, s.len - a.d.window) : 0;
  s.base = s.lo & ~(kTile - 1);
  s.blocks = (s.len - s.base + kBlock - 1) / kBlock;
  return s;
}

// Exchanges halves: the low (or high) 16 bits of two registers.
__device__ __forceinline__ uint32_t low_halves(uint32_t a, uint32_t b) { return __builtin_amdgcn_perm(b, a, 0x05040100u); }
__device__ __forceinline__ uint32_t high_halves(uint32_t a, uint32_t b) { return __builtin_amdgcn_perm(b, a, 0x07060302u); }

__device__ __forceinline__ f32x4 mfma_bf16(u32x4 a, u32x4 b, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}
__device__ __forceinline__ f32x4 mfma_f32(float a, float b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x4f32(a, b, c, 0, 0, 0); }

// One wave's operands for head vectors of up to DP values (a multiple of 64; D are there, the others are zeros).  A lane is
// (j = lane / 16, n = lane % 16).
//   key piece i of a token: its 16 bytes at byte 64 i + 16 j;  a lane's columns of V: columns(c) for c < DP / 16
template <bool kBf16, int DP>
struct Tile {
  static constexpr int kSize = kBf16 ? 2 : 4;
  static constexpr int kKeyPieces = DP * kSize / 64;
  static constexpr int kCols = DP / 16;                         // of V, a lane
  static constexpr int kValuePieces = kCols * kSize / 16 > 0 ? kCols * kSize / 16 : 1;  // of 16 bytes (one of 8 if that is less)
  static constexpr bool kHalfPiece = kCols * kSize == 8;

  struct Keys {
    u32x4 of[2][kKeyPieces];
  };
  u32x4 val[8][kValuePieces];

  // Byte of a row where the lane's piece p of V begins.
  static __device__ __forceinline__ int value_byte(int p, int n) { return kBf16 ? n * kCols * 2 + 16 * p : 256 * p + 16 * n; }
  // Column of V that element c of the lane n's operands stands for.
  static __device__ __forceinline__ int column(int c, int n) { return kBf16 ? n * kCols + c : 64 * (c / 4) + 4 * n + c % 4; }

  static __device__ __forceinline__ void load_key(Keys &keys, int half, const char *row, int j, int bytes) {
#pragma unroll
    for (int i = 0; i < kKeyPieces; ++i) {
      const int at = 64 * i + 16 * j;
      u32x4 q = {0u, 0u, 0u, 0u};
      if (at < bytes) q = *reinterpret_cast<const u32x4 *>(row + at);
      keys.of[half][i] = q;
    }
  }
  template <bool kOnce>
  __device__ __forceinline__ void load_value(int i, const char *row, int n, int bytes) {
#pragma unroll
    for (int p = 0; p < kValuePieces; ++p) {
      const int at = value_byte(p, n);
      u32x4 q = {0u, 0u, 0u, 0u};
      if (at < bytes) {
        if (kHalfPiece) {
          const u32x2 h = kOnce ? __builtin_nontemporal_load(reinterpret_cast<const u32x2 *>(row + at)) : *reinterpret_cast<const u32x2 *>(row + at);
          q[0] = h[0];
          q[1] = h[1];
        } else {
          q = kOnce ? __builtin_nontemporal_load(reinterpret_cast<const u32x4 *>(row + at)) : *reinterpret_cast<const u32x4 *>(row + at);
        }
      }
      val[i][p] = q;
    }
  }
  __device__ __forceinline__ void clear_value(int i) {
#pragma unroll
    for (int p = 0; p < kValuePieces; ++p) val[i][p] = u32x4{0u, 0u, 0u, 0u};
  }

  static __device__ __forceinline__ f32x4 scores(const Keys &keys, int half, const u32x4 (&query)[kKeyPieces]) {
    f32x4 s = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < kKeyPieces; ++i) {
      if (kBf16) {
        s = mfma_bf16(keys.of[half][i], query[i], s);
      } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) s = mfma_f32(__uint_as_float(keys.of[half][i][e]), __uint_as_float(query[i][e]), s);
      }
    }
    return s;
  }
  // O^T += V^T P^T; p: the lane's eight tokens
  __device__ __forceinline__ void add(const float (&p)[8], f32x4 (&o)[kCols]) const {
    if (kBf16) {
      u32x4 pb;
#pragma unroll
      for (int i = 0; i < 4; ++i) pb[i] = pack2(p[2 * i], p[2 * i + 1]);
#pragma unroll
      for (int c = 0; c < kCols; ++c) {
        u32x4 a;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const uint32_t x = val[2 * i][c / 8][(c / 2) % 4], y = val[2 * i + 1][c / 8][(c / 2) % 4];
          a[i] = c % 2 == 0 ? low_halves(x, y) : high_halves(x, y);
        }
        o[c] = mfma_bf16(a, pb, o[c]);
      }
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i)
#pragma unroll
        for (int c = 0; c < kCols; ++c) o[c] = mfma_f32(__uint_as_float(val[i][c / 4][c % 4]), p[i], o[c]);
    }
  }
};

constexpr int waves_a_simd(bool bf16, int dp) { return dp == 256 ? 1 : 2; }

// a / b of which one, as a rule, does not need 64 bits.
__device__ __forceinline__ int64_t quotient64(int64_t n, int64_t d) {
  return (n | d) >> 32 == 0 ? static_cast<int64_t>(static_cast<uint32_t>(n) / static_cast<uint32_t>(d)) : n / d;
}
__device__ __forceinline__ int64_t run_of(const StepArgs &a, int64_t total) { return quotient64(total + a.workgroups - 1, a.workgroups); }

// kOnce: values go past the caches.
template <bool kBf16, int DP, int kWaves, bool kDealt, bool kOnce>
__global__ __launch_bounds__(64 * kWaves, waves_a_simd(kBf16, DP)) void step_kernel(const StepArgs a) {
  using T = Tile<kBf16, DP>;
  // keys are asked for a tile ahead where that costs no wave, or where there is none to lose
  constexpr bool kAhead = kDealt ? kBf16 && DP == 256 : kWaves == 8 ? kBf16 || DP == 64 : kBf16 && DP != 128;
  __shared__ union {
    Prefix prefix;
    struct {
      float o[kWaves][kRows][DP + 4];
      float m[kWaves][kRows], l[kWaves][kRows];
    } join;
  } lds;
  const int lane = threadIdx.x & 63, wave = threadIdx.x / 64, j = lane / 16, n = lane % 16;
  const int rows_of_heads = a.d.G, bytes = a.d.D * T::kSize;
  const int64_t page_bytes = (static_cast<int64_t>(a.d.Hk) << a.d.lg_page) * bytes;
  const int page_mask = (1 << a.d.lg_page) - 1;

  // the run of this workgroup, and where it begins
  int64_t left_of_run = 0;
  int b, unit, block = 0;
  Span sp;
  if (kDealt) {
    int64_t left;
    if (a.d.B <= 64) {  // a wave has them all
      int blocks = lane < a.d.B ? span_of(a, lane).blocks : 0, sum = blocks;  // (2^24 each at most)
#pragma unroll
      for (int k = 1; k < 64; k <<= 1) {
        const int o = __shfl_up(sum, k);
        if (lane >= k) sum += o;
      }
      const int64_t total = static_cast<int64_t>(__builtin_amdgcn_readlane(sum, 63)) * a.units;
      const int64_t run = run_of(a, total), at = blockIdx.x * run;
      left_of_run = min(run, total - at);
      if (left_of_run <= 0) return;
      b = __builtin_popcountll(__ballot(static_cast<int64_t>(sum) * a.units <= at));
      left = at - static_cast<int64_t>(__builtin_amdgcn_readlane(sum - blocks, b)) * a.units;
      sp = span_of(a, b);
    } else {
      count_blocks(lds.prefix, a.d.B, [&](int i) { return span_of(a, i).blocks; });
      const int64_t total = uniform(lds.prefix.at[kDealers]) * a.units;
      const int64_t run = run_of(a, total), at = blockIdx.x * run;
      left_of_run = min(run, total - at);
      if (left_of_run <= 0) return;
      const int dealer = dealer_of(lds.prefix, at, a.units);
      b = dealer * share_of(a.d.B);
      left = uniform(at - lds.prefix.at[dealer] * a.units);
      sp = span_of(a, b);
      while (left >= static_cast<int64_t>(sp.blocks) * a.units) {
        left -= static_cast<int64_t>(sp.blocks) * a.units;
        sp = span_of(a, ++b);
      }
      __syncthreads();
    }
    unit = static_cast<int>(quotient64(left, sp.blocks));
    block = static_cast<int>(left - static_cast<int64_t>(unit) * sp.blocks);
  } else {
    b = static_cast<int>(blockIdx.x / static_cast<unsigned>(a.units));
    unit = static_cast<int>(blockIdx.x) - b * a.units;
    sp = span_of(a, b);
  }
  bool continued = block > 0;

  while (true) {
    const int blocks = kDealt ? static_cast<int>(min(static_cast<int64_t>(sp.blocks - block), left_of_run)) : sp.blocks;
    const int hk = unit / a.row_tiles, first_row = (unit - hk * a.row_tiles) * kRows;
    const int rows = min(kRows, rows_of_heads - first_row);
    const int64_t row0 = static_cast<int64_t>(b) * a.d.H + hk * a.d.G + first_row;  // of q and y
    const int32_t *table = a.table + static_cast<int64_t>(b) * a.d.max_pages;
    const char *kh = static_cast<const char *>(a.k) + (static_cast<int64_t>(hk) << a.d.lg_page) * bytes;
    const char *vh = static_cast<const char *>(a.v) + (static_cast<int64_t>(hk) << a.d.lg_page) * bytes;

    u32x4 query[T::kKeyPieces];
#pragma unroll
    for (int i = 0; i < T::kKeyPieces; ++i) {
      const int byte = 64 * i + 16 * j;
      query[i] = u32x4{0u, 0u, 0u, 0u};
      if (n < rows && byte < bytes)
        query[i] = *reinterpret_cast<const u32x4 *>(static_cast<const char *>(a.q) + (row0 + n) * bytes + byte);
    }
    f32x4 o[T::kCols];
#pragma unroll
    for (int c = 0; c < T::kCols; ++c) o[c] = f32x4{0.f, 0.f, 0.f, 0.f};
    float m = kNone, l = 0.f;

    // pages of tokens n and 16 + n of a tile (tokens that aren't seen: of the nearest one that is)
    struct Pages {
      int of[2];
    };
    auto pages_of = [&](int first) {
      Pages p;
#pragma unroll
      for (int h = 0; h < 2; ++h) p.of[h] = table[min(max(first + 16 * h + n, sp.lo), sp.len - 1) >> a.d.lg_page];
      return p;
    };
    auto there = [&](int page) { return static_cast<unsigned>(page) < static_cast<unsigned>(a.d.npages); };
    auto load_keys = [&](typename T::Keys &keys, int first, const Pages &p) {
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int token = min(max(first + 16 * h + n, sp.lo), sp.len - 1);
        T::load_key(keys, h, kh + (there(p.of[h]) ? p.of[h] : 0) * page_bytes + (token & page_mask) * bytes, j, bytes);
      }
    };
    int first = sp.base + block * kBlock + wave * kTile;
    const int last = min(sp.len, sp.base + (block + blocks) * kBlock);
    typename T::Keys keys_ahead;
    Pages pages_ahead, pages_next;
    if (kAhead && first < last) {
      pages_ahead = pages_of(first);
      load_keys(keys_ahead, first, pages_ahead);
      pages_next = pages_of(first + kWaves * kTile);
    }
    for (; first < last; first += kWaves * kTile) {
      T t;
      typename T::Keys keys;
      Pages pages;
      if (kAhead) {
        keys = keys_ahead;
        pages = pages_ahead;
      } else {
        pages = pages_of(first);
        load_keys(keys, first, pages);
      }
      uint32_t seen = 0xffffffffu;
      if (first < sp.lo) seen &= 0xffffffffu << (sp.lo - first);
      if (first + kTile > sp.len) seen &= 0xffffffffu >> (first + kTile - sp.len);
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        seen &= ~(static_cast<uint32_t>(__ballot(!there(pages.of[h])) & 0xffffu) << (16 * h));
        if (!there(pages.of[h])) pages.of[h] = 0;
      }
      if (a.d.lg_page >= 2) {  // four neighbouring tokens of an aligned tile are on one page
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const int64_t where = __shfl(pages.of[h], 4 * j) * page_bytes;
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            const int token = min(max(first + 16 * h + 4 * j + r, sp.lo), sp.len - 1);
            const int64_t row = token >> 2 == (first + 16 * h + 4 * j) >> 2 ? where + (token & page_mask) * bytes : where;
            t.template load_value<kOnce>(4 * h + r, vh + row, n, bytes);
          }
        }
      } else {
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            const int token = min(max(first + 16 * h + 4 * j + r, sp.lo), sp.len - 1);
            t.template load_value<kOnce>(4 * h + r, vh + __shfl(pages.of[h], 4 * j + r) * page_bytes + (token & page_mask) * bytes, n, bytes);
          }
      }
      if (kAhead) {  // (behind the last tile: the last token's, not used)
        load_keys(keys_ahead, first + kWaves * kTile, pages_next);
        pages_ahead = pages_next;
        pages_next = pages_of(first + 2 * kWaves * kTile);
      }
      f32x4 s[2];
#pragma unroll
      for (int h = 0; h < 2; ++h) s[h] = T::scores(keys, h, query);
      if (seen != 0xffffffffu) {  // (what isn't seen may hold anything: no product with it is kept)
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
          for (int r = 0; r < 4; ++r)
            if (!((seen >> (16 * h + 4 * j + r)) & 1u)) {
              s[h][r] = -INFINITY;
              t.clear_value(4 * h + r);
            }
      }
      float top = fmaxf(fmaxf(fmaxf(s[0][0], s[0][1]), fmaxf(s[0][2], s[0][3])), fmaxf(fmaxf(s[1][0], s[1][1]), fmaxf(s[1][2], s[1][3])));
      top = fmaxf(top, __shfl_xor(top, 16));
      top = fmaxf(top, __shfl_xor(top, 32));
      top *= a.scale_log2;
      if (__any(top > m)) {
        const float next = fmaxf(m, fminf(top, kMost)), keep = __builtin_amdgcn_exp2f(m - next);
        m = next;
        l *= keep;
#pragma unroll
        for (int c = 0; c < T::kCols; ++c)
#pragma unroll
          for (int r = 0; r < 4; ++r) o[c][r] *= keep;
      }
      float p[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        p[i] = __builtin_amdgcn_exp2f(fmaf(s[i / 4][i % 4], a.scale_log2, -m));  // (rounded at the difference's size, not the logit's)
        l += p[i];
      }
      t.add(p, o);
    }
    l += __shfl_xor(l, 16);
    l += __shfl_xor(l, 32);

    // join the waves
    if (j == 0) {
      lds.join.m[wave][n] = m;
      lds.join.l[wave][n] = l;
    }
#pragma unroll
    for (int r = 0; r < 4; ++r)
#pragma unroll
      for (int c = 0; c < T::kCols; c += 4) {
        const f32x4 q = {o[c][r], o[c + 1][r], o[c + 2][r], o[c + 3][r]};
        *reinterpret_cast<f32x4 *>(&lds.join.o[wave][n][T::column(c, 4 * j + r)]) = q;
      }
    __syncthreads();
    const bool whole = !kDealt || blocks == sp.blocks;
    if (kDealt && threadIdx.x == 0) {
      Spread &spread = a.spread[static_cast<int64_t>(b) * a.units + unit];
      if (!continued) spread.first = static_cast<int>(blockIdx.x);
      if (block + blocks == sp.blocks) spread.last = static_cast<int>(blockIdx.x);
    }
    const int slot_row = (2 * static_cast<int>(blockIdx.x) + (continued ? 0 : 1)) * kRows;
    for (int e = threadIdx.x; e < rows * (DP / 4); e += 64 * kWaves) {
      const int row = e / (DP / 4), col = (e % (DP / 4)) * 4;
      if (col >= a.d.D) continue;
      float top = kNone, f[kWaves], sum = 0.f;
#pragma unroll
      for (int w = 0; w < kWaves; ++w) top = fmaxf(top, lds.join.m[w][row]);
      f32x4 v = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int w = 0; w < kWaves; ++w) {
        f[w] = __builtin_amdgcn_exp2f(lds.join.m[w][row] - top);
        sum = fmaf(lds.join.l[w][row], f[w], sum);
        const f32x4 ow = *reinterpret_cast<const f32x4 *>(&lds.join.o[w][row][col]);
#pragma unroll
        for (int r = 0; r < 4; ++r) v[r] = fmaf(ow[r], f[w], v[r]);
      }
      if (whole) {
        const float inv = sum == 0.f ? 0.f : 1.f / sum;
        if (kBf16) {
          const u32x2 q = {pack2(v[0] * inv, v[1] * inv), pack2(v[2] * inv, v[3] * inv)};
          *reinterpret_cast<u32x2 *>(static_cast<uint16_t *>(a.y) + (row0 + row) * a.d.D + col) = q;
        } else {
          const f32x4 q = {v[0] * inv, v[1] * inv, v[2] * inv, v[3] * inv};
          *reinterpret_cast<f32x4 *>(static_cast<float *>(a.y) + (row0 + row) * a.d.D + col) = q;
        }
      } else {
        float *part = a.part + static_cast<int64_t>(slot_row + row) * (a.d.D + 4);
        *reinterpret_cast<f32x4 *>(part + col) = v;
        if (col == 0) {
          part[a.d.D] = top;
          part[a.d.D + 1] = sum;
        }
      }
    }
    left_of_run -= blocks;
    if (!kDealt || left_of_run <= 0) break;
    __syncthreads();
    block = 0;
    continued = false;
    if (++unit == a.units) {
      unit = 0;
      do sp = span_of(a, ++b);
      while (sp.blocks == 0);
    }
  }
}

// Joins what the workgroups of a unit left.  A workgroup takes `rows` heads and `cols` pieces of four values of a unit, and as many
// of the parts at a time as it has threads for.
template <bool kBf16>
__global__ __launch_bounds__(kThreads) void join_kernel(const StepArgs a, int rows, int cols, int row_cuts, int col_cuts) {
  constexpr int kAhead = 2;  // parts whose values are on their way at a time
  struct Share {
    f32x4 o;
    float m, l;
  };
  __shared__ Share got[kThreads];
  const auto join = [](float &top, float &sum, f32x4 &v, float m, float l, f32x4 o) {
    const float next = fmaxf(top, m), keep = __builtin_amdgcn_exp2f(top - next), f = __builtin_amdgcn_exp2f(m - next);
    top = next;
    sum = fmaf(sum, keep, l * f);
#pragma unroll
    for (int r = 0; r < 4; ++r) v[r] = fmaf(v[r], keep, o[r] * f);
  };
  unsigned id = blockIdx.x;
  const int col_cut = static_cast<int>(id % col_cuts), row_cut = static_cast<int>(id / col_cuts % row_cuts);
  id /= static_cast<unsigned>(col_cuts * row_cuts);
  const int b = static_cast<int>(id / static_cast<unsigned>(a.units)), unit = static_cast<int>(id) - b * a.units;
  const Spread spread = a.spread[id];
  const int hk = unit / a.row_tiles, first_row = (unit - hk * a.row_tiles) * kRows;
  const int64_t row0 = static_cast<int64_t>(b) * a.d.H + hk * a.d.G + first_row;
  const int row_end = min(min(kRows, a.d.G - first_row), (row_cut + 1) * rows), col_end = min(a.d.D / 4, (col_cut + 1) * cols);
  int first = 0, last = -1;
  if (span_of(a, b).blocks > 0) {  // (otherwise nobody has been there)
    first = spread.first;
    last = spread.last;
    if (first == last) return;  // finished where it was computed
  }
  const int items = rows * cols, abreast = max(1, kThreads / items);
  for (int e0 = 0; e0 < items; e0 += kThreads) {
    const int e = e0 + (items < kThreads ? threadIdx.x % items : threadIdx.x), lane = items < kThreads ? threadIdx.x / items : 0;
    const int row = row_cut * rows + e / cols, col = 4 * (col_cut * cols + e % cols);
    const bool mine = e < items && lane < abreast && row < row_end && col < 4 * col_end;
    float top = kNone, sum = 0.f;
    f32x4 v = {0.f, 0.f, 0.f, 0.f};
    if (mine) {
      for (int w0 = first + lane; w0 <= last; w0 += kAhead * abreast) {
        float m[kAhead], l[kAhead];
        f32x4 o[kAhead];
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
          const int w = w0 + i * abreast;
          m[i] = kNone;
          l[i] = 0.f;
          o[i] = f32x4{0.f, 0.f, 0.f, 0.f};
          if (w <= last) {
            const float *part = a.part + static_cast<int64_t>((2 * w + (w == first ? 1 : 0)) * kRows + row) * (a.d.D + 4);
            m[i] = part[a.d.D];
            l[i] = part[a.d.D + 1];
            o[i] = *reinterpret_cast<const f32x4 *>(part + col);
          }
        }
#pragma unroll
        for (int i = 0; i < kAhead; ++i) join(top, sum, v, m[i], l[i], o[i]);
      }
    }
    if (abreast > 1) {
      Share &mine_of = got[threadIdx.x];
      mine_of.m = top;
      mine_of.l = sum;
      mine_of.o = v;
      for (int d = 1 << (31 - __builtin_clz(abreast - 1)); d > 0; d >>= 1) {
        __syncthreads();
        if (mine && lane < d && lane + d < abreast) {
          const Share &other = got[threadIdx.x + d * items];
          join(top, sum, v, other.m, other.l, other.o);
          mine_of.m = top;
          mine_of.l = sum;
          mine_of.o = v;
        }
      }
    }
    if (mine && lane == 0) {
      const float inv = sum == 0.f ? 0.f : 1.f / sum;
      if (kBf16) {
        const u32x2 q = {pack2(v[0] * inv, v[1] * inv), pack2(v[2] * inv, v[3] * inv)};
        *reinterpret_cast<u32x2 *>(static_cast<uint16_t *>(a.y) + (row0 + row) * a.d.D + col) = q;
      } else {
        const f32x4 q = {v[0] * inv, v[1] * inv, v[2] * inv, v[3] * inv};
        *reinterpret_cast<f32x4 *>(static_cast<float *>(a.y) + (row0 + row) * a.d.D + col) = q;
      }
    }
  }
}

// Whether work is dealt, from the most tokens that a sequence can have: half of them are reckoned with.  In us, with 32 heads over
// 8 of 128, bf16: a unit to a workgroup takes 4 and its bytes at 52 GB/s, or all units' at 6 TB/s; dealing takes 9 and all units'
// bytes at 5.2 TB/s, and is charged 3 more, for lengths that are alike lose more by it than uneven ones win.  One sequence of 518
// tokens: 8.8 and 9.9 dealt; of 2000: 22 and 10; 16 of 2000: 23 and 30.  A sequence of more than a MiB a key head, 20 us for a
// workgroup, may be the only one that long: then work is dealt.
bool dealt(const AttnDims &d) {
  const double tokens = d.window > 0 ? std::min(d.capacity(), d.window) : d.capacity();
  const double longest = 2.0 * tokens * d.D * (d.bf16 ? 2 : 4), all = 0.5 * longest * d.B * units_of(d);
  if (longest > 1048576.0) return true;
  return 4.0 + std::max(longest / 52.0e3, all / 6.0e6) > 12.0 + all / 5.2e6;
}

// A unit to a workgroup: of eight waves where there is a CU for each; of four otherwise, of which two or three share a CU, so that
// the start of one is beside the others' work.  32 heads over 8 of 128, bf16: 16 sequences of 500 tokens 9.1 us and 12.5, 64 of 250
// 15.0 and 12.5, of 1000 41.7 and 38.7, 1024 of 1 to 200 134 and 52.
//
// Caches that do not fit the last-level cache (256 MiB; the rule takes 320 of the caches, since the host does not know what is used
// of them; what was measured nearest is 125 and 500 MiB) have been pushed out of it by the time they are read again: there, values, of
// which an instruction reads whole lines, are loaded as data of no further use, and leave room for the keys, of which one reads half
// lines.  64 sequences to 32768 165 us and 150, 16 of 8000 103 and 84; with caches that fit 16 of 2000 23 and 27.  (Both so: 16 of 8000
// 90.)
template <bool kBf16, int DP, bool kOnce>
void launch_step(const StepArgs &a, hipStream_t stream) {
  constexpr int kWide = DP <= 128 ? 8 : 4;  // waves: two a SIMD, where registers allow
  const unsigned units = static_cast<unsigned>(a.units) * a.d.B;
  if (dealt(a.d))
    hipLaunchKernelGGL((step_kernel<kBf16, DP, kThreads / 64, true, kOnce>), dim3(a.workgroups), dim3(kThreads), 0, stream, a);
  else if (units <= kCUs)
    hipLaunchKernelGGL((step_kernel<kBf16, DP, kWide, false, false>), dim3(units), dim3(64 * kWide), 0, stream, a);
  else
    hipLaunchKernelGGL((step_kernel<kBf16, DP, 4, false, kOnce>), dim3(units), dim3(256), 0, stream, a);
}
template <bool kBf16, int DP>
void launch_step(const StepArgs &a, hipStream_t stream) {
  const double caches = 2.0 * a.d.npages * (static_cast<double>(a.d.Hk) * (1 << a.d.lg_page)) * a.d.D * (kBf16 ? 2 : 4);
  if (caches > 335544320.0) launch_step<kBf16, DP, true>(a, stream);
  else launch_step<kBf16, DP, false>(a, stream);
}

// The joining launch.  Few units have many parts each, up to one of every workgroup: a workgroup for 32 values of a head.  Otherwise one
// for half the heads.
struct Join {
  int rows, cols, row_cuts, col_cuts;
  int64_t workgroups;
};
Join join_of(const AttnDims &d) {
  const int64_t units = static_cast<int64_t>(units_of(d)) * d.B;
  const int tile_rows = d.G < kRows ? d.G : kRows, all_cols = d.D / 4;
  const bool few = units < kFewUnits;
  Join j;
  j.rows = few ? 1 : (tile_rows + 1) / 2;
  j.cols = few && all_cols > 8 ? 8 : all_cols;
  j.row_cuts = (tile_rows + j.rows - 1) / j.rows;
  j.col_cuts = (all_cols + j.cols - 1) / j.cols;
  j.workgroups = units * j.row_cuts * j.col_cuts;
  return j;
}

template <bool kBf16>
hipError_t launch(const StepArgs &a, hipStream_t stream) {
  if (a.d.D <= 64) launch_step<kBf16, 64>(a, stream);
  else if (a.d.D <= 128) launch_step<kBf16, 128>(a, stream);
  else launch_step<kBf16, 256>(a, stream);
  if (const hipError_t e = hipGetLastError(); e != hipSuccess || !dealt(a.d)) return e;
  const Join j = join_of(a.d);
  hipLaunchKernelGGL(join_kernel<kBf16>, dim3(static_cast<unsigned>(j.workgroups)), dim3(kThreads), 0, stream, a, j.rows, j.cols, j.row_cuts, j.col_cuts);
  return hipGetLastError();
}

size_t part_bytes(const AttnDims &d) { return (static_cast<size_t>(2 * kMostWorkgroups * kRows) * (d.D + 4) * 4 + 255) / 256 * 256; }

}  // namespace

bool attn_step_fits(const AttnDims &d) {
  return dealt(d) ? join_of(d).workgroups <= kMostWorkgroups256 : static_cast<int64_t>(units_of(d)) * d.B <= kMostWorkgroups256;
}

size_t attn_step_used_bytes(const AttnDims &d) {
  if (!dealt(d)) return 256;
  return part_bytes(d) + (static_cast<size_t>(d.B) * units_of(d) * sizeof(Spread) + 255) / 256 * 256;
}
size_t attn_step_workspace_bytes(const AttnDims &d) {
  AttnDims one = d;  // (dealt's two sides come closer with every sequence: if it deals the work of some, then that of one)
  one.B = 1;
  if (!dealt(one)) return 256;
  return part_bytes(d) + (static_cast<size_t>(d.B) * units_of(d) * sizeof(Spread) + 255) / 256 * 256;
}

hipError_t launch_attn_step(const AttnDims &d, const int32_t *lens, const int32_t *table, const void *q, const void *k_cache,
                            const void *v_cache, float scale, void *y, void *workspace, hipStream_t stream) {
  StepArgs a = {};
  a.lens = lens;
  a.table = table;
  a.q = q;
  a.k = k_cache;
  a.v = v_cache;
  a.y = y;
  a.part = static_cast<float *>(workspace);
  a.spread = reinterpret_cast<Spread *>(static_cast<char *>(workspace) + part_bytes(d));
  a.d = d;
  a.row_tiles = row_tiles_of(d);
  a.units = units_of(d);
  a.workgroups = workgroups_of(d.bf16, d.D <= 64 ? 64 : d.D <= 128 ? 128 : 256);
  a.scale_log2 = scale * 1.44269504f;
  return d.bf16 ? launch<true>(a, stream) : launch<false>(a, stream);
}

}  // namespace ssd
