// Causal attention of packed new tokens over a paged cache:  y[t][h] = sum_s softmax_s(scale q[t][h] . K[s]) V[s], s up to t's
// position.
//
// Bound by the matrix pipe for prompts, by the pass over K and V for a few new tokens behind a long cache.  The rows of a unit
// are 128 (token, head) pairs of one sequence and key head, tokens slowest, so that a key head's query heads share its K and V;
// a wave has 32 of them as the columns of 32 x 32 matrix products and keeps their running maximum m, sum l and O^T in registers:
//
//   S^T (tokens x rows) = K Q^T,   p = 2^(S - m),   O^T (values x rows) += V^T P^T
//
// Tiles of K and V (64 tokens; fp32: 32) go through LDS, the next one being on its way while one is worked on.  fp32 is taken apart
// into three values of bf16 each, and six products stand for one.  The first product leaves a lane with tokens 8i + 4h .. 8i + 4h + 3
// (h = lane / 32) of its row; these are what it supplies as the second operand of V^T P^T, whose first operand comes from LDS by
// transposing reads, with the same order of tokens.
//
// Where there are few units, several workgroups share one's tokens and leave (m, l, O) in the workspace for a second launch.
//
// 32 heads over 8 of 128, bf16: 16384 tokens 2.04 to 2.19 ms from card to card, 1000 to 1080 TFLOP/s of the causal products (the
// library's large product: 1316); 4096 tokens 148 us, 1024 tokens 26 us; 64 tokens behind 32000 55 us.  fp32: see its kernel.
#include <algorithm>
#include <cmath>

#include "ssd_attn.hpp"
#include "ssd_split_bf16.hpp"

namespace ssd {
namespace {

using namespace block;

constexpr int kWaves = 4, kThreads = 64 * kWaves, kWaveRows = 32, kUnitRows = kWaves * kWaveRows;
constexpr int kWorkgroups = 256;  // of eight waves, which fill the GPU
constexpr int kManyUnits = 768;   // from so many on, a unit is for one group of four waves, and not shared
constexpr int kManyTiles = 16;    // two groups of waves are for units of so many tiles,
constexpr int kFewTiles = 6;      // of so many where there is a CU for each unit
constexpr int kMostSplits = 64;   // of a unit
// Where units are shared, a workgroup is to have a little more than its part of all tiles.  A unit has less than twice its
// sequence's average of them, so that there are at most 2 kWorkgroups / 1.25 workgroups more than units.
constexpr float kShare = 1.25f / kWorkgroups;
constexpr int kMostParts = 2 * kWorkgroups;
constexpr float kLongShare = 64.f;  // tiles, from which on the number of rounds is looked at
// A maximum of nothing: finite, so that differences are numbers.  None is larger than its opposite: behind that, probabilities are
// infinite and y is not a number, where those of an infinite maximum would all be zero.
constexpr float kNone = -3.0e38f;
constexpr int tokens_of_tile(bool bf16) { return bf16 ? 64 : 32; }
// Tiles that a workgroup at least takes where several share a unit, in us 5 in bf16 and 8 in fp32 with heads of 128 values alone on
// a CU: fewer cost more in parts than they save.  (bf16, 3 tokens behind 27000, 8 heads over 1, window 927: 15 us, with 8 tiles 18; 90
// pieces of 0 to 6 tokens behind up to 2000, 16 heads over 2: 28.6 and 26.7.)
inline int least_tiles(const AttnDims &d) { return d.bf16 ? 5 : d.D <= 128 ? 4 : 2; }
// There is no search for the largest score of a step: the sum of a lane's probabilities, which is needed anyway, says whether one is
// too large for the running maximum.  Until then they are up to this (bf16, 16384 tokens: 2.07 ms, a search for every step 2.28).
// bf16: what is summed are the probabilities as they are rounded for their product with the values, so that the rounding of a token
// that outweighs the others drops out: error against 64 bits, 24 rows that see 920 tokens, logits of deviation 2, in units of the
// result's rounding: 1.30 on average and 1.48 at most of 150 draws, with exact sums 1.40 and 1.81.
constexpr float kMost = 256.f;

// A unit as the joining launch needs it; each workgroup leaves one, with splits = 0 if it is not the first of a shared unit.
struct Record {
  int rows, first_row, begin, splits;
};

struct PrefillArgs {
  const int32_t *cu, *lens, *table;
  const void *q, *k, *v;
  void *y;
  void *part;        // of each workgroup
  Record *record;    // likewise
  AttnDims d;
  uint32_t inv_group;
  int units;         // at most, of a key head
  int splits;        // at most, of a unit
  int least;         // tiles of a split
  int parts;         // there is room for
  int groups;        // of waves, a workgroup (bf16)
  float scale_log2;  // scale * log2(e)
};

// A unit's rows and the tokens they see; one of the workgroups that share it.
struct Unit {
  int rows;        // 0: there is no such unit
  int first_row;   // of its sequence
  int seq, begin;  // the sequence and its first new token
  int pos0;        // that token's position
  int base, tiles, splits;
  int split;       // this workgroup's
};
template <int kTokens>
__device__ __forceinline__ void see(const PrefillArgs &a, Unit &r) {
  const int lowest = r.pos0 + quotient(r.first_row, a.d.G, a.inv_group);
  const int highest = min(r.pos0 + quotient(r.first_row + r.rows - 1, a.d.G, a.inv_group), a.d.capacity() - 1);
  r.base = (a.d.window > 0 ? max(0, lowest + 1 - a.d.window) : 0) & ~(kTokens - 1);
  r.tiles = highest < max(0, lowest) ? 0 : (highest + 1 - r.base + kTokens - 1) / kTokens;
}
// What this lane's row sees, and its wave's 32 rows, whose positions do not decrease.
struct Seen {
  int from, to;                  // the row: [from, to]
  int all_from, all_to;          // of the wave: every row sees [all_from, all_to],
  int any_from, any_to;          // none sees what is not in [any_from, any_to]
  __device__ __forceinline__ Seen(const PrefillArgs &a, int pos) {
    const int capacity = a.d.capacity(), lowest = __builtin_amdgcn_readfirstlane(pos), highest = __builtin_amdgcn_readlane(pos, 31);
    // (a token behind the row of the page table has no place, and sees nothing)
    to = pos < capacity ? pos : -1;
    from = a.d.window > 0 ? pos - a.d.window + 1 : 0;
    all_from = __builtin_amdgcn_readlane(from, 31);
    any_from = __builtin_amdgcn_readfirstlane(from);
    all_to = highest < capacity ? lowest : -1;
    any_to = highest < capacity ? highest : lowest < capacity ? capacity - 1 : -1;
  }
};
// A sequence's units.
struct Line {
  int begin, pos0, all;  // all: rows
  int units, tiles;      // tiles of the last unit, which has the most (rows behind the page table's row have none)
  float work;            // tiles of all, about
};
template <int kTokens>
__device__ __forceinline__ Line line_of(const PrefillArgs &a, int b) {
  Line r = {};
  if (b >= a.d.B) return r;
  r.begin = min(max(a.cu[b], 0), a.d.T);
  const int count = min(max(a.cu[b + 1], 0), a.d.T) - r.begin;
  r.pos0 = max(a.lens[b], 0) - count;
  if (count <= 0) return r;
  r.all = count * a.d.G;
  r.units = (r.all - 1) / kUnitRows + 1;
  Unit u = {};
  u.pos0 = r.pos0;
  u.rows = min(kUnitRows, r.all);
  see<kTokens>(a, u);
  const int first_tiles = u.tiles;
  u.first_row = (r.units - 1) * kUnitRows;
  u.rows = r.all - u.first_row;
  see<kTokens>(a, u);
  r.tiles = max(first_tiles, u.tiles);
  r.work = 0.5f * static_cast<float>(r.units) * static_cast<float>(first_tiles + r.tiles);
  return r;
}
__device__ __forceinline__ int splits_of(const PrefillArgs &a, float tiles, float share) {
  return min(max(static_cast<int>(ceilf(tiles / share)), 1), a.splits);
}
__device__ __forceinline__ int64_t shuffle_up64(int64_t v, int k) {
  const int lo = __shfl_up(static_cast<int>(v), k), hi = __shfl_up(static_cast<int>(v >> 32), k);
  return static_cast<int64_t>(hi) << 32 | static_cast<uint32_t>(lo);
}
// Where workgroups have much to do and there are more than CUs, the number that a CU gets one after the other decides.  A lane
// reckons for the longest unit shared by as many workgroups as the lane's number and one: how many rounds those make which have
// about the most to do, and what the parts cost, in tiles.  (It takes 3 us.)  32 heads over 8 of 128: 640 tokens behind 30000 484 us
// without this and 357 with, twice 300 behind 8000 144 and 115; four times 156 behind 32000, 25 heads over 5, 510 and 394.
__device__ __forceinline__ float best_share(const PrefillArgs &a, const Line &line, int lanes, float load, float share) {
  const int lane = threadIdx.x & 63;
  int longest = line.tiles, simply = line.units * splits_of(a, static_cast<float>(line.tiles), share);
#pragma unroll 1
  for (int d = 1; d < lanes; d <<= 1) {
    longest = max(longest, __shfl_xor(longest, d));
    simply += __shfl_xor(simply, d);
  }
  if (__builtin_amdgcn_readfirstlane(simply) * a.d.Hk <= kWorkgroups) return share;
  const float tiles_of_longest = 1.0001f * static_cast<float>(__builtin_amdgcn_readfirstlane(longest));
  const float mine = fmaxf(tiles_of_longest / static_cast<float>(lane + 1), static_cast<float>(a.least));
  int all = 0, front = 0;
#pragma unroll 1
  for (int b = 0; b < lanes; ++b) {
    const int units = __builtin_amdgcn_readlane(line.units, b);
    const float tiles = static_cast<float>(__builtin_amdgcn_readlane(line.tiles, b));
    const int splits = splits_of(a, tiles, mine);
    all += units * splits;
    if (2.f * tiles > mine * static_cast<float>(splits)) front += units * splits;
  }
  const float cost = fmaxf(ceilf(static_cast<float>(front * a.d.Hk) * (1.f / kWorkgroups)) * mine, load) + 0.04f * static_cast<float>(all * a.d.Hk);
  // (the least of them, with its lane in the last bits)
  uint32_t least = all * a.d.Hk > a.parts ? 0xffffffffu : (__float_as_uint(cost) & ~63u) | static_cast<uint32_t>(lane);
#pragma unroll 1
  for (int d = 1; d < 64; d <<= 1) least = min(least, static_cast<uint32_t>(__shfl_xor(static_cast<int>(least), d)));
  least = __builtin_amdgcn_readfirstlane(least);
  return least == 0xffffffffu ? share : fmaxf(tiles_of_longest / static_cast<float>((least & 63u) + 1u), static_cast<float>(a.least));
}
// The unit of workgroup k of a key head, in the order in which they are begun: the sequences whose workgroups have the most
// tiles first, of a sequence the last units first, which see the most tokens.  A long unit is shared by as many workgroups as give
// each a little more than the average CU's load, which only the device knows.  They have neighbouring numbers, and there are no
// gaps but where a prompt's first units need fewer: a workgroup without work that is between others leaves its CU idle for as long
// as theirs take.  Every wave finds out by itself, a lane a sequence.  (Many sequences, whose units are many and not shared, are not
// gone through: 1024 of 4 tokens behind 200, 32 heads over 8: 232 us, gone through in order 432.)  Ten pieces of 0 to 512 tokens behind up to 20000, 20 heads over
// 4, window 4096: 63 us, with units in the order of the sequences and the same shares for all 71; eight prompts of 1 to 4096 tokens,
// 16 heads over 4: 141 and 153.
template <int kTokens>
__device__ __forceinline__ Unit find_unit(const PrefillArgs &a, int k) {
  const int lane = threadIdx.x & 63, lanes = min(a.d.B, 64);
  Unit r = {};
  if (a.splits == 1 && a.d.B > 64) {
    // Sequence b's units are counted from cu[b] * group / rows + b on: these are at least as far apart as its units are many.
    const int u = a.units - 1 - k;
    const auto first_unit = [&](int b) { return static_cast<int64_t>(min(max(a.cu[b], 0), a.d.T)) * a.d.G / kUnitRows + b; };
    int low = 0, high = a.d.B;  // the last one that does not begin behind u is in [low, high)
    while (high - low > 1) {
      const int step = (high - low + 63) / 64, b = low + lane * step;
      const uint64_t m = __ballot(b < high && first_unit(b) <= u);
      if (m == 0) return r;
      low += (63 - __builtin_clzll(m)) * step;
      high = min(high, low + step);
    }
    low = __builtin_amdgcn_readfirstlane(low);
    const Line line = line_of<kTokens>(a, low);
    const int64_t place = u - first_unit(low);
    if (place < 0 || place >= line.units) return r;
    r.seq = low;
    r.begin = line.begin;
    r.pos0 = line.pos0;
    r.splits = 1;
    r.first_row = static_cast<int>(place) * kUnitRows;
    r.rows = min(kUnitRows, line.all - r.first_row);
    see<kTokens>(a, r);
    return r;
  }
  Line line = line_of<kTokens>(a, lane);
  float share = 0.f;  // tiles that a workgroup is to have
  if (a.splits > 1) {
    float work = line.work;
    for (int b0 = 64; b0 < a.d.B; b0 += 64) work += line_of<kTokens>(a, b0 + lane).work;
    for (int d = 1; d < lanes; d <<= 1) work += __shfl_xor(work, d);
    work = __uint_as_float(__builtin_amdgcn_readfirstlane(__float_as_uint(work)));
    share = fmaxf(work * static_cast<float>(a.d.Hk) * kShare, static_cast<float>(a.least));
    if (a.d.B <= 64 && share > kLongShare) share = best_share(a, line, lanes, work * static_cast<float>(a.d.Hk) / kWorkgroups, share);
  }
  int done = 0;  // workgroups of the sequences in front of these 64
  for (int b0 = 0; b0 < a.d.B; b0 += 64) {
    if (b0 > 0) line = line_of<kTokens>(a, b0 + lane);
    const int splits = a.splits > 1 ? splits_of(a, static_cast<float>(line.tiles), share) : 1;
    const int n = line.units * splits, per = line.tiles / splits;
    int most = per;
    for (int d = 1; d < lanes; d <<= 1) most = max(most, __shfl_xor(most, d));
    const bool front = 2 * per > most;
    // workgroups of those in front in the upper half, of the others in the lower one
    const int64_t mine = front ? static_cast<int64_t>(n) << 32 : n;
    int64_t sum = mine;
    for (int d = 1; d < lanes; d <<= 1) {
      const int64_t o = shuffle_up64(sum, d);
      if (lane >= d) sum += o;
    }
    const int fronts = __builtin_amdgcn_readlane(static_cast<int>(sum >> 32), lanes - 1);
    const int first = done + (front ? static_cast<int>((sum - mine) >> 32) : fronts + static_cast<int>(sum - mine));
    const uint64_t here = __ballot(k >= first && k < first + n);
    if (here != 0) {
      const int l = __builtin_ctzll(here);
      const auto of = [&](int v) { return __builtin_amdgcn_readlane(v, l); };
      r.seq = b0 + l;
      r.begin = of(line.begin);
      r.pos0 = of(line.pos0);
      r.splits = of(splits);
      const int place = k - of(first), u = place / r.splits;
      r.split = place - u * r.splits;
      r.first_row = (of(line.units) - 1 - u) * kUnitRows;
      r.rows = min(kUnitRows, of(line.all) - r.first_row);
      see<kTokens>(a, r);
      r.splits = max(1, min(r.splits, (r.tiles + a.least - 1) / a.least));
      if (r.split >= r.splits) r.rows = 0;
      return r;
    }
    done += __builtin_amdgcn_readlane(static_cast<int>(sum >> 32) + static_cast<int>(sum), lanes - 1);
  }
  return r;
}

__device__ __forceinline__ f32x16 mfma_bf16(u32x4 a, u32x4 b, f32x16 c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}

// Transposed LDS read (ds_read_b64_tr_b16): in each group of 16 lanes, lane i names four neighbouring 16-bit values, of row i / 4
// and columns 4 (i % 4) on, and receives column i of the four rows.
__device__ __forceinline__ u32x2 lds_transposed(const char *p) {
  typedef short s16x4 __attribute__((ext_vector_type(4)));
  typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
  return __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)(uint32_t)(uintptr_t)p));
}

// The same from a constant offset behind the lane's address.
__device__ __forceinline__ u32x2 lds_transposed(uint32_t lane_at, int offset) {
  typedef short s16x4 __attribute__((ext_vector_type(4)));
  typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
  typedef __attribute__((address_space(3))) char lds_char;
  return __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)((lds_char *)lane_at + offset)));
}

__device__ __forceinline__ uint32_t lds_address(const void *p) { return static_cast<uint32_t>(reinterpret_cast<uintptr_t>(p)); }
// 16 bytes from each lane's address to LDS, in the order of the lanes from `to` (of the wave) on.  An LDS read behind it in the
// program does not wait for it: that is for the one who reads.
__device__ __forceinline__ void load_to_lds(const void *from, uint32_t to) {
  asm volatile("s_mov_b32 m0, %1\n\ts_nop 4\n\tglobal_load_lds_dwordx4 %0, off" : : "v"(from), "s"(to) : "m0", "memory");
}
// The same from a lane's offset behind the wave's address.
__device__ __forceinline__ void load_to_lds(const void *wave_from, uint32_t offset, uint32_t to) {
  asm volatile("s_mov_b32 m0, %2\n\ts_nop 4\n\tglobal_load_lds_dwordx4 %0, %1" : : "v"(offset), "s"(wave_from), "s"(to) : "m0", "memory");
}

// Geometry of a bf16 tile in LDS for head vectors of up to DP values (D are there, the others are zeros): rows of kPieces pieces of
// 16 bytes, in an order that depends on the row so that the reads of either product go to all banks.
template <int DP>
struct Geometry {
  static constexpr int kTokens = tokens_of_tile(true);
  static constexpr int kRowBytes = 2 * DP, kPieces = kRowBytes / 16;
  static constexpr int kTileBytes = kTokens * kRowBytes;
  static constexpr int kFetch = kTokens * kPieces / kThreads;  // pieces of a tile a thread brings
  // 16 lanes read the same piece of neighbouring rows
  static __device__ __forceinline__ int key_piece(int row, int c) { return c ^ (row & (kPieces < 16 ? kPieces - 1 : 15)); }
  // 32 lanes read 64 bytes of four neighbouring rows
  static __device__ __forceinline__ int value_piece(int row, int c) { return DP == 64 ? c ^ ((row & 2) << 1) : c ^ ((row & 3) << 2); }
};

// A part of a unit as its four waves hold it, lane by lane: the pieces of O^T, four columns of the lane's row each, then m and l.
template <int DP>
struct Part {
  static constexpr int kPieces = DP / 8;
  f32x4 o[kWaves][kPieces][64];
  float m[kWaves][64], l[kWaves][64];
};

// Four columns of a row, of O / l, to y.
template <bool kBf16>
__device__ __forceinline__ void write_row(const PrefillArgs &a, int64_t out_row, int col, f32x4 o, float inv) {
  if (col >= a.d.D) return;
  if constexpr (kBf16) {
    const u32x2 q = {pack2(o[0] * inv, o[1] * inv), pack2(o[2] * inv, o[3] * inv)};
    *reinterpret_cast<u32x2 *>(static_cast<uint16_t *>(a.y) + out_row * a.d.D + col) = q;
  } else {
    const f32x4 q = {o[0] * inv, o[1] * inv, o[2] * inv, o[3] * inv};
    *reinterpret_cast<f32x4 *>(static_cast<float *>(a.y) + out_row * a.d.D + col) = q;
  }
}
// Piece i of a lane: columns 8 i + 4 h on of its row (o: columns 32 c + 8 (r / 4) + 4 h + r % 4).
__device__ __forceinline__ int piece_column(int i, int h) { return 8 * i + 4 * h; }

// A wave's rows' end: to y, or as a part to the workspace.
template <bool kBf16, int DP>
__device__ __forceinline__ void finish(const PrefillArgs &a, bool whole, int slot, bool mine, int wave, int64_t out_row, const f32x16 (&o)[DP / 32],
                                       float m, float l) {
  const int lane = threadIdx.x & 63, h = lane / 32;
  const float inv = l == 0.f ? 0.f : 1.f / l;
  Part<DP> *const part = static_cast<Part<DP> *>(a.part) + slot;
#pragma unroll
  for (int i = 0; i < Part<DP>::kPieces; ++i) {
    const f32x4 q = {o[i / 4][4 * (i % 4)], o[i / 4][4 * (i % 4) + 1], o[i / 4][4 * (i % 4) + 2], o[i / 4][4 * (i % 4) + 3]};
    if (!whole) part->o[wave][i][lane] = q;
    else if (mine) write_row<kBf16>(a, out_row, piece_column(i, h), q, inv);
  }
  if (!whole) {
    part->m[wave][lane] = m;
    part->l[wave][lane] = l;
  }
}

// A workgroup may have two groups of four waves, each with every second tile of a unit.  Joins the second one's results to the
// first one's; false for the second group, which is done then.
template <int DP>
__device__ __forceinline__ bool join_groups(Part<DP> &part, int group, int wave, f32x16 (&o)[DP / 32], float &m, float &l) {
  const int lane = threadIdx.x & 63;
  if (group == 1) {
#pragma unroll
    for (int i = 0; i < Part<DP>::kPieces; ++i)
      part.o[wave][i][lane] = f32x4{o[i / 4][4 * (i % 4)], o[i / 4][4 * (i % 4) + 1], o[i / 4][4 * (i % 4) + 2], o[i / 4][4 * (i % 4) + 3]};
    part.m[wave][lane] = m;
    part.l[wave][lane] = l;
  }
  __syncthreads();
  if (group == 1) return false;
  const float other = part.m[wave][lane], top = fmaxf(m, other), keep = __builtin_amdgcn_exp2f(m - top), f = __builtin_amdgcn_exp2f(other - top);
  m = top;
  l = fmaf(l, keep, part.l[wave][lane] * f);
#pragma unroll
  for (int i = 0; i < Part<DP>::kPieces; ++i) {
    const f32x4 q = part.o[wave][i][lane];
#pragma unroll
    for (int r = 0; r < 4; ++r) o[i / 4][4 * (i % 4) + r] = fmaf(o[i / 4][4 * (i % 4) + r], keep, q[r] * f);
  }
  return true;
}

// c and the two bf16 values of a register.
__device__ __forceinline__ float add_both(uint32_t two, float c) {
  typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
  return __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, two), __builtin_bit_cast(bf16x2, 0x3f803f80u), c, false);
}

// Rows that see nothing of a part keep no product with what others see.
template <int kColTiles>
__device__ __forceinline__ void clear_unseen(f32x16 (&o)[kColTiles], float l) {
  if (!__any(l == 0.f)) return;
#pragma unroll
  for (int c = 0; c < kColTiles; ++c)
#pragma unroll
    for (int r = 0; r < 16; ++r) o[c][r] = l == 0.f ? 0.f : o[c][r];
}

// The larger of the two values that lanes l and l + 32 hold, in both.
__device__ __forceinline__ float both_halves_max(float v) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}

// The kernel of bf16.  Step by step, 32 tokens at a time, with a product between each request to LDS and its use: the scores of
// the next step are computed beside the softmax of this one, and its values read meanwhile; the keys of the step behind that are
// read before this step's product with the values.  Tiles come to LDS straight from memory, one barrier a tile.  Two workgroups
// share a CU, two waves a SIMD.
template <int DP, bool kFull, int kGroups>
__global__ __launch_bounds__(kThreads * kGroups, DP == 256 ? 1 : 2) void prefill_bf16_kernel(const PrefillArgs a) {
  using Geo = Geometry<DP>;
  constexpr int kTokens = Geo::kTokens, kColTiles = DP / 32, kFetch = Geo::kFetch;
  constexpr int kSteps = kTokens / 32;               // of a tile
  constexpr int kPieces = DP / 16;                   // of a query row, a lane
  constexpr bool kEarly = DP <= 128;                 // registers are there for reads from LDS ahead of their use
  constexpr int kPassRows = kThreads / Geo::kPieces; // rows of a tile that the workgroup brings at a time,
  constexpr int kWaveLoadRows = kPassRows / kWaves;  // and a wave of it
  constexpr int kKeyTiles = kEarly ? 2 : 3;
  __shared__ __align__(16) char lds[kGroups][kKeyTiles + 2][Geo::kTileBytes];
  static_assert(kGroups == 1 || sizeof(Part<DP>) <= sizeof(lds));

  const int hk = static_cast<int>(blockIdx.x) % a.d.Hk;
  const Unit unit = find_unit<kTokens>(a, static_cast<int>(blockIdx.x) / a.d.Hk);
  if (a.splits > 1 && threadIdx.x == 0)
    a.record[blockIdx.x] = Record{unit.rows, unit.first_row, unit.begin, unit.rows > 0 && unit.split == 0 && unit.splits > 1 ? unit.splits : 0};
  if (unit.rows == 0) return;

  const int lane = threadIdx.x & 63, n = lane & 31, h = lane / 32;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64) % kWaves, group = __builtin_amdgcn_readfirstlane(threadIdx.x / 64) / kWaves;
  const int thread = 64 * wave + lane;  // of the group
  char (*const lds_k)[Geo::kTileBytes] = lds[group], (*const lds_v)[Geo::kTileBytes] = lds[group] + kKeyTiles;
  const int bytes = kFull ? DP * 2 : a.d.D * 2;
  const uint32_t page_bytes = static_cast<uint32_t>(a.d.Hk * bytes) << a.d.lg_page;
  const int page_mask = (1 << a.d.lg_page) - 1;
  const int32_t *table = a.table + static_cast<int64_t>(unit.seq) * a.d.max_pages;

  // this lane's row
  const int local = wave * 32 + n;
  const bool mine = local < unit.rows;
  const int row = unit.first_row + min(local, unit.rows - 1), token = quotient(row, a.d.G, a.inv_group);
  const Seen seen(a, unit.pos0 + token);
  const int64_t out_row = static_cast<int64_t>(unit.begin + token) * a.d.H + hk * a.d.G + (row - token * a.d.G);
  u32x4 query[kPieces];
#pragma unroll
  for (int i = 0; i < kPieces; ++i) {
    const int byte = 32 * i + 16 * h;
    query[i] = u32x4{0u, 0u, 0u, 0u};
    if (mine && byte < bytes) query[i] = *reinterpret_cast<const u32x4 *>(static_cast<const char *>(a.q) + out_row * bytes + byte);
  }
  const bool idle = wave * 32 >= unit.rows;

  // the split's tiles, of which the group takes every kGroups-th
  const int tile1 = static_cast<int>(static_cast<int64_t>(unit.tiles) * (unit.split + 1) / unit.splits);
  const int tile0 = static_cast<int>(static_cast<int64_t>(unit.tiles) * unit.split / unit.splits) + group;
  const int rounds = (tile1 - (tile0 - group) + kGroups - 1) / kGroups;
  const int end = min(unit.pos0 + quotient(unit.first_row + unit.rows - 1, a.d.G, a.inv_group) + 1, a.d.capacity());  // tokens seen by any row

  // ---- bringing tiles: memory to LDS, a piece a lane; lane t of a wave knows the page of the tile's token t ----
  const int my_row = thread / Geo::kPieces, my_slot = thread % Geo::kPieces;
  const char *const kh = static_cast<const char *>(a.k) + (static_cast<int64_t>(hk) << a.d.lg_page) * bytes;
  const char *const vh = static_cast<const char *>(a.v) + (static_cast<int64_t>(hk) << a.d.lg_page) * bytes;
  if (!kFull) {  // the pieces that no row has
    for (int i = thread; i < (kKeyTiles + 2) * Geo::kTileBytes / 16; i += kThreads) reinterpret_cast<u32x4 *>(lds[group])[i] = u32x4{0u, 0u, 0u, 0u};
    __syncthreads();
  }
  // (for a token behind the last one that is seen: the page of that one)
  auto page_of = [&](int tile) { return table[min(unit.base + tile * kTokens + lane, end - 1) >> a.d.lg_page]; };
  // where a wave's loads of a tile begin in either cache, if they are on one page each
  struct Where {
    uint64_t at[kFetch];
  };
  auto where_of = [&](int tile, int page) {
    Where w;
    const int tile_first = unit.base + tile * kTokens;
    const int there = static_cast<unsigned>(page) < static_cast<unsigned>(a.d.npages) ? page : 0;
#pragma unroll
    for (int i = 0; i < kFetch; ++i) {
      const int at = wave * kWaveLoadRows + i * kPassRows;
      w.at[i] = static_cast<uint64_t>(static_cast<uint32_t>(__builtin_amdgcn_readlane(there, at))) * page_bytes +
                static_cast<uint32_t>(((tile_first + at) & page_mask) * bytes);
    }
    return w;
  };
  const bool one_page = page_mask >= kWaveLoadRows - 1;
  auto bring = [&](char *to, const char *head, const Where &w, int tile, int page, bool keys) {
    const uint32_t to_wave = __builtin_amdgcn_readfirstlane(lds_address(to)) + wave * 1024;
    if (one_page) {
#pragma unroll
      for (int i = 0; i < kFetch; ++i) {
        const int row = my_row + (kPassRows % 16 == 0 ? 0 : i * kPassRows);
        const int piece = keys ? Geo::key_piece(row, my_slot) : Geo::value_piece(row, my_slot);
        if (kFull || 16 * piece < bytes)
          load_to_lds(head + w.at[i], static_cast<uint32_t>((lane / Geo::kPieces) * bytes + 16 * piece), to_wave + i * kThreads * 16);
      }
      return;
    }
    const int there = static_cast<unsigned>(page) < static_cast<unsigned>(a.d.npages) ? page : 0;
#pragma unroll
    for (int i = 0; i < kFetch; ++i) {
      const uint32_t where = __shfl(there, my_row + i * kPassRows);
      const int row = my_row + i * kPassRows, piece = keys ? Geo::key_piece(row, my_slot) : Geo::value_piece(row, my_slot);
      const uint32_t in_page = ((unit.base + tile * kTokens + row) & page_mask) * bytes + 16 * piece;
      if (kFull || 16 * piece < bytes) load_to_lds(head + (static_cast<uint64_t>(where) * page_bytes + in_page), to_wave + i * kThreads * 16);
    }
  };
  // tokens of a tile that are seen by no row: behind the last one, or of a page that is not in the cache
  auto gone_of = [&](int tile, int page) {
    const int first = unit.base + tile * kTokens;
    return __ballot(lane < kTokens && (static_cast<unsigned>(page) >= static_cast<unsigned>(a.d.npages) || first + lane >= end));
  };
  // (their probability is zero, and so must be its product: once the values are there, zeros take their place)
  auto arrived = [&](char *values, uint64_t gone) {
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    if (gone != 0) {
#pragma unroll
      for (int i = 0; i < kFetch; ++i)
        if ((gone >> (my_row + i * kPassRows)) & 1) *reinterpret_cast<u32x4 *>(values + 16 * thread + i * kThreads * 16) = u32x4{0u, 0u, 0u, 0u};
    }
    __syncthreads();
  };

  f32x16 o[kColTiles];
  float m = kNone, l = 0.f;
#pragma unroll
  for (int c = 0; c < kColTiles; ++c)
#pragma unroll
    for (int r = 0; r < 16; ++r) o[c][r] = 0.f;
  // addresses in a tile
  const int k_row = n * Geo::kRowBytes;
  const int v_row = (lane & 15) / 4, v_byte = 32 * ((lane >> 4) & 1) + 8 * (lane & 3);  // (8 bytes of a 64-byte column tile)
  u32x4 keys[kPieces];  // of the step whose scores come next
  auto read_keys = [&](const char *tile, int step) {
#pragma unroll
    for (int i = 0; i < kPieces; ++i)
      keys[i] = *reinterpret_cast<const u32x4 *>(tile + 32 * step * Geo::kRowBytes + k_row + 16 * Geo::key_piece(n, 2 * i + h));
  };
  auto scores = [&](const char *tile, int step) {
    f32x16 to;
#pragma unroll
    for (int r = 0; r < 16; ++r) to[r] = 0.f;
    if (!kEarly) read_keys(tile, step);
#pragma unroll
    for (int i = 0; i < kPieces; ++i) to = mfma_bf16(keys[i], query[i], to);
    return to;
  };

  // The keys of a step are read two steps ahead, those of the tile in work with the one before it: in LDS are, of the tile in
  // work, its values, and of the next one the keys.
  uint64_t gone[3] = {0, 0, 0};       // of the tile in work and the next two
  int page_k = 0;                     // of the tile whose keys are asked for next
  Where where_v = {};                 // of the tile whose values are asked for next
  int page_v = 0;
  if (rounds > 0) {
    const int p0 = page_of(tile0), p1 = page_of(tile0 + kGroups);
    page_v = p1;
    page_k = page_of(tile0 + 2 * kGroups);
    gone[0] = gone_of(tile0, p0);
    gone[1] = gone_of(tile0 + kGroups, p1);
    const Where w0 = where_of(tile0, p0);
    where_v = where_of(tile0 + kGroups, p1);
    bring(lds_k[0], kh, w0, tile0, p0, true);
    bring(lds_v[0], vh, w0, tile0, p0, false);
    bring(lds_k[1], kh, where_v, tile0 + kGroups, p1, true);
  }
  arrived(lds_v[0], gone[0]);
  int at_k = 0, round = 0;
  const auto wrap = [](int i) { return i >= kKeyTiles ? i - kKeyTiles : i; };
  // the next tile's values and the keys of the one behind it
  const auto bring_next = [&](char *kt2, char *vt1) {
    const int tile = tile0 + kGroups * round;
    // (tiles behind the last one repeat its last token: they are brought and not used)
    const Where where_k = where_of(tile + 2 * kGroups, page_k);
    bring(vt1, vh, where_v, tile + kGroups, page_v, false);
    bring(kt2, kh, where_k, tile + 2 * kGroups, page_k, true);
    gone[2] = gone_of(tile + 2 * kGroups, page_k);
    where_v = where_k;
    page_v = page_k;
    page_k = page_of(tile + 3 * kGroups);
  };
  const auto next_round = [&](char *vt1) {
    gone[0] = gone[1];
    gone[1] = gone[2];
    at_k = wrap(at_k + 1);
    arrived(vt1, gone[0]);
  };
  f32x16 s;
  const auto begin = [&](const char *tile) {
    if (kEarly) read_keys(tile, 0);
    s = scores(tile, 0);
    if (kEarly) read_keys(tile, 1);
  };
  // Tiles in front of all that the wave's rows see are brought for the other waves, and left out here: their values may be
  // anything, infinities included.  (32 tokens at a time, behind the rows too, by a branch in the loop: 4 % more time.)
  const int skipped = min(max(0, (seen.any_from - unit.base) / kTokens - tile0 + kGroups - 1) / kGroups, rounds);
  if (kEarly && skipped == 0) begin(lds_k[0]);
  __syncthreads();
#pragma unroll 1
  for (; round < skipped; ++round) {
    char *const vt1 = lds_v[(round & 1) ^ 1];
    bring_next(lds_k[wrap(at_k + 2)], vt1);
    if (kEarly && round + 1 == skipped) begin(lds_k[wrap(at_k + 1)]);
    next_round(vt1);
  }
  if (!kEarly) begin(lds_k[at_k]);
  for (; round < rounds; ++round) {
    const int tile = tile0 + kGroups * round;
    const int first = unit.base + tile * kTokens;
    char *const kt = lds_k[at_k], *const kt1 = lds_k[wrap(at_k + 1)], *const kt2 = lds_k[wrap(at_k + 2)];
    char *const vt = lds_v[round & 1], *const vt1 = lds_v[(round & 1) ^ 1];
    bring_next(kt2, vt1);
    if (!idle && tile < tile1 && first <= seen.any_to) {
#pragma unroll
      for (int step = 0; step < kSteps; ++step) {
        if (first + 32 * step + 31 > seen.all_to || first + 32 * step < seen.all_from || gone[0] != 0) {
          asm volatile("" ::: "memory");  // (nothing of this is computed where the branch isn't taken)
          const uint32_t out = static_cast<uint32_t>(gone[0] >> (32 * step)) >> (4 * h);
          const int to = seen.to - (first + 32 * step + 4 * h), from = seen.from - (first + 32 * step + 4 * h);
#pragma unroll
          for (int r = 0; r < 16; ++r) {
            const int t = 8 * (r / 4) + r % 4;
            if (t > to || t < from || (out & (1u << t))) s[r] = -INFINITY;
          }
        }
        u32x4 p[2];
        float sum;
        auto exponentials = [&] {
          float sums[2] = {0.f, 0.f};
#pragma unroll
          for (int r = 0; r < 8; r += 2)
#pragma unroll
            for (int g = 0; g < 2; ++g) {
              const float x = __builtin_amdgcn_exp2f(fmaf(s[8 * g + r], a.scale_log2, -m)), y = __builtin_amdgcn_exp2f(fmaf(s[8 * g + r + 1], a.scale_log2, -m));
              p[g][r / 2] = pack2(x, y);
              sums[g] = add_both(p[g][r / 2], sums[g]);
            }
          sum = sums[0] + sums[1];
        };
        // the values of the step, by groups of 16 tokens and 32 columns
        const char *const v_lane = vt + (32 * step + 4 * h + v_row) * Geo::kRowBytes;
        auto read_values = [&](int g, int c) {
          const char *const v_at = v_lane + 16 * g * Geo::kRowBytes + 16 * Geo::value_piece(v_row, 4 * c + v_byte / 16) + v_byte % 16;
          const u32x2 lo = lds_transposed(v_at), hi = lds_transposed(v_at + 8 * Geo::kRowBytes);
          return u32x4{lo[0], lo[1], hi[0], hi[1]};
        };
        u32x4 values[2][kEarly ? kColTiles : 1];
        if (kEarly)
#pragma unroll
          for (int g = 0; g < 2; ++g)
#pragma unroll
            for (int c = 0; c < kColTiles; ++c) values[g][kEarly ? c : 0] = read_values(g, c);
        __builtin_amdgcn_s_setprio(1);
        const f32x16 next = scores(step + 1 < kSteps ? kt : kt1, step + 1 < kSteps ? step + 1 : 0);
        exponentials();
        __builtin_amdgcn_s_setprio(0);
        if (__any(!(sum <= kMost))) {
          asm volatile("" ::: "memory");
          float top = s[0];
#pragma unroll
          for (int r = 1; r < 16; ++r) top = fmaxf(top, s[r]);
          const float larger = fmaxf(m, fminf(both_halves_max(top) * a.scale_log2, -kNone)), keep = __builtin_amdgcn_exp2f(m - larger);
          m = larger;
          l *= keep;
#pragma unroll
          for (int c = 0; c < kColTiles; ++c)
#pragma unroll
            for (int r = 0; r < 16; ++r) o[c][r] *= keep;
          exponentials();
        }
        l += sum;
        if (kEarly) read_keys(kt1, step);
#pragma unroll
        for (int g = 0; g < 2; ++g)
#pragma unroll
          for (int c = 0; c < kColTiles; ++c) o[c] = mfma_bf16(kEarly ? values[g][kEarly ? c : 0] : read_values(g, c), p[g], o[c]);
        s = next;
      }
    }
    next_round(vt1);
  }
  l += __shfl_xor(l, 32);
  clear_unseen(o, l);
  if (kGroups == 2 && !join_groups<DP>(*reinterpret_cast<Part<DP> *>(lds), group, wave, o, m, l)) return;
  finish<true, DP>(a, unit.splits == 1, blockIdx.x, mine, wave, out_row, o, m, l);
}

// Groups of waves of a workgroup.  Heads of up to 64 values: three workgroups share a CU, and what each does on the vector ALU is
// beside the others' products (8192 tokens, 16 heads: 745 us, with two groups 760; 1023 tokens, 12 heads: 27 and 31).  Up to 128:
// two waves a SIMD is what registers allow, and two groups finish a unit sooner than one (2048 tokens, 16 heads, twice: 206 and 301).
constexpr int f32_groups(int dp) { return dp == 128 ? 2 : 1; }
// The kernel of fp32, on bf16 products too: a value is the sum of three of bf16, and six products of parts stand for one (what is
// left out is 2^-24 of it, an fp32 product's rounding), at 16 times the rate of fp32's own.  A tile is taken apart once, on its way
// to LDS; the next one waits in registers meanwhile.  Probabilities are taken apart as they are made.  Against fp32's own
// instruction: 1023 tokens, 12 heads over 4 of 64: 27 us and 41; 8192 tokens, 16 over 4 of 64: 745 and 1180; 2048 tokens, 16 over 4 of
// 128, twice: 206 and 327; of 256, once: 311 and 424.
template <int DP>
__global__ __launch_bounds__(kThreads * f32_groups(DP), DP == 256 ? 1 : 2) void prefill_f32_kernel(const PrefillArgs a) {
  using split::Op;
  constexpr bool kEarly = DP <= 64;  // registers are there for the next tile during the keys' product
  constexpr int kTokens = tokens_of_tile(false), kColTiles = DP / 32, kGroups = f32_groups(DP);
  constexpr int kSteps = DP / 16;                        // of a product with a key
  constexpr int kFetch = kTokens * DP / 8 / kThreads;    // pieces of 8 values of a tile that a thread brings
  // Rows of a part in LDS, so far apart that a read's go to all banks: 16 bytes of neighbouring rows (K), 64 of four (V)
  constexpr int kKeyRow = 2 * DP + 16, kValueRow = 2 * DP + 64, kPieces = DP / 8;
  constexpr int kKeyPart = kTokens * kKeyRow, kValuePart = kTokens * kValueRow;
  __shared__ __align__(16) char all_lds[kGroups][3 * kKeyPart + 3 * kValuePart];
  static_assert(kGroups == 1 || sizeof(Part<DP>) <= sizeof(all_lds));

  const int hk = static_cast<int>(blockIdx.x) % a.d.Hk;
  const Unit unit = find_unit<kTokens>(a, static_cast<int>(blockIdx.x) / a.d.Hk);
  if (a.splits > 1 && threadIdx.x == 0)
    a.record[blockIdx.x] = Record{unit.rows, unit.first_row, unit.begin, unit.rows > 0 && unit.split == 0 && unit.splits > 1 ? unit.splits : 0};
  if (unit.rows == 0) return;

  const int lane = threadIdx.x & 63, n = lane & 31, h = lane / 32;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64) % kWaves, group = __builtin_amdgcn_readfirstlane(threadIdx.x / 64) / kWaves;
  const int thread = 64 * wave + lane;  // of the group
  char *const lds_k = all_lds[group], *const lds_v = lds_k + 3 * kKeyPart;
  const int bytes = a.d.D * 4;
  const int64_t page_bytes = (static_cast<int64_t>(a.d.Hk) << a.d.lg_page) * bytes;
  const int page_mask = (1 << a.d.lg_page) - 1;
  const char *kh = static_cast<const char *>(a.k) + (static_cast<int64_t>(hk) << a.d.lg_page) * bytes;
  const char *vh = static_cast<const char *>(a.v) + (static_cast<int64_t>(hk) << a.d.lg_page) * bytes;
  const int32_t *table = a.table + static_cast<int64_t>(unit.seq) * a.d.max_pages;

  // this lane's row
  const int local = wave * kWaveRows + n;
  const bool mine = local < unit.rows;
  const int row = unit.first_row + min(local, unit.rows - 1), token = quotient(row, a.d.G, a.inv_group);
  const Seen seen(a, unit.pos0 + token);
  const int64_t out_row = static_cast<int64_t>(unit.begin + token) * a.d.H + hk * a.d.G + (row - token * a.d.G);
  const bool idle = wave * kWaveRows >= unit.rows;

  auto take_apart = [](const u32x4 (&q)[2], Op (&o)[3]) {
    float v[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = __uint_as_float(q[e / 4][e % 4]);
    split::split3_even(v, o);
  };
  Op query[kSteps][3];
#pragma unroll
  for (int i = 0; i < kSteps; ++i) {
    const int byte = 64 * i + 32 * h;
    u32x4 q[2] = {u32x4{0u, 0u, 0u, 0u}, u32x4{0u, 0u, 0u, 0u}};
    if (mine && byte < bytes) {
      const u32x4 *from = reinterpret_cast<const u32x4 *>(static_cast<const char *>(a.q) + out_row * bytes + byte);
      q[0] = from[0];
      q[1] = from[1];
    }
    take_apart(q, query[i]);
  }
  f32x16 o[kColTiles];
#pragma unroll
  for (int c = 0; c < kColTiles; ++c)
#pragma unroll
    for (int r = 0; r < 16; ++r) o[c][r] = 0.f;
  float m = kNone, l = 0.f;

  // the split's tiles, of which the group takes every kGroups-th
  const int tile1 = static_cast<int>(static_cast<int64_t>(unit.tiles) * (unit.split + 1) / unit.splits);
  const int tile0 = static_cast<int>(static_cast<int64_t>(unit.tiles) * unit.split / unit.splits) + group;
  const int rounds = (tile1 - (tile0 - group) + kGroups - 1) / kGroups;
  const int end = min(unit.pos0 + quotient(unit.first_row + unit.rows - 1, a.d.G, a.inv_group) + 1, a.d.capacity());  // tokens seen by any row

  u32x4 fetched[2][kFetch][2];
  uint64_t gone = 0, gone_next = 0;  // tokens of the tile whose page is not in the cache
  auto page_of = [&](int tile) { return table[min(unit.base + tile * kTokens + (lane & (kTokens - 1)), end - 1) >> a.d.lg_page]; };
  auto fetch = [&](int tile, int page) {
    const int first = unit.base + tile * kTokens;
    const bool bad = static_cast<unsigned>(page) >= static_cast<unsigned>(a.d.npages);
    gone_next = __ballot(bad) & ((1ull << kTokens) - 1);
    if (bad) page = -1;
#pragma unroll
    for (int i = 0; i < kFetch; ++i) {
      const int piece = thread + i * kThreads, r = piece / kPieces, c = piece % kPieces;
      const int where = __shfl(page, r);
      const int at = min(first + r, end - 1) & page_mask;
#pragma unroll
      for (int e = 0; e < 2; ++e) fetched[0][i][e] = fetched[1][i][e] = u32x4{0u, 0u, 0u, 0u};
      // (a token behind the last one that is seen is brought as zeros: its probability is zero, and so must be the product)
      if (where >= 0 && 32 * c < bytes && first + r < end) {
        const int64_t byte = where * page_bytes + static_cast<int64_t>(at) * bytes + 32 * c;
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          fetched[0][i][e] = *reinterpret_cast<const u32x4 *>(kh + byte + 16 * e);
          fetched[1][i][e] = *reinterpret_cast<const u32x4 *>(vh + byte + 16 * e);
        }
      }
    }
  };
  auto stage = [&] {
#pragma unroll
    for (int i = 0; i < kFetch; ++i) {
      const int piece = thread + i * kThreads, r = piece / kPieces, c = piece % kPieces;
      Op parts[3];
      take_apart(fetched[0][i], parts);
#pragma unroll
      for (int p = 0; p < 3; ++p) *reinterpret_cast<u32x4 *>(lds_k + p * kKeyPart + r * kKeyRow + 16 * c) = parts[p].q;
      take_apart(fetched[1][i], parts);
#pragma unroll
      for (int p = 0; p < 3; ++p) *reinterpret_cast<u32x4 *>(lds_v + p * kValuePart + r * kValueRow + 16 * c) = parts[p].q;
    }
    gone = gone_next;
  };
  const char *const k_lane = lds_k + n * kKeyRow + 16 * h;
  const uint32_t v_lane = lds_address(lds_v + (4 * h + (lane & 15) / 4) * kValueRow + 32 * ((lane >> 4) & 1) + 8 * (lane & 3));

  if (rounds > 0) {
    fetch(tile0, page_of(tile0));
    stage();
  }
  __syncthreads();
  for (int round = 0; round < rounds; ++round) {
    const int tile = tile0 + kGroups * round, first = unit.base + tile * kTokens;
    const uint64_t gone_now = gone;
    const bool busy = !idle && tile < tile1 && first <= seen.any_to && first + kTokens > seen.any_from;
    const int page_next = page_of(tile + kGroups);
    if (kEarly && round + 1 < rounds) fetch(tile + kGroups, page_next);
    f32x16 s;
    if (busy) {
#pragma unroll
      for (int r = 0; r < 16; ++r) s[r] = 0.f;
      Op k[2][3];
      auto read_keys = [&](int i) {
#pragma unroll
        for (int p = 0; p < 3; ++p) k[i & 1][p].q = *reinterpret_cast<const u32x4 *>(k_lane + p * kKeyPart + 32 * i);
      };
      read_keys(0);
#pragma unroll
      for (int i = 0; i < kSteps; ++i) {
        if (i + 1 < kSteps) read_keys(i + 1);
        s = split::mfma6(k[i & 1], query[i], s);
        if (DP > 64) asm volatile("" ::: "memory");  // (no reads further ahead: there are no registers for them)
      }
      if (first + kTokens - 1 > seen.all_to || first < seen.all_from || gone_now != 0) {
        asm volatile("" ::: "memory");  // (nothing of this is computed where the branch isn't taken)
        const uint32_t out = static_cast<uint32_t>(gone_now) >> (4 * h);
        const int to = seen.to - (first + 4 * h), from = seen.from - (first + 4 * h);
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          const int t = 8 * (r / 4) + r % 4;
          if (t > to || t < from || (out & (1u << t))) s[r] = -INFINITY;
        }
      }
      float e[16], sum;
      auto exponentials = [&] {
        sum = 0.f;
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          e[r] = __builtin_amdgcn_exp2f(fmaf(s[r], a.scale_log2, -m));
          sum += e[r];
        }
      };
      exponentials();
      if (__any(!(sum <= kMost))) {
        asm volatile("" ::: "memory");
        float top = s[0];
#pragma unroll
        for (int r = 1; r < 16; ++r) top = fmaxf(top, s[r]);
        const float larger = fmaxf(m, fminf(both_halves_max(top) * a.scale_log2, -kNone)), keep = __builtin_amdgcn_exp2f(m - larger);
        m = larger;
        l *= keep;
#pragma unroll
        for (int c = 0; c < kColTiles; ++c)
#pragma unroll
          for (int r = 0; r < 16; ++r) o[c][r] *= keep;
        exponentials();
      }
      l += sum;
#pragma unroll
      for (int r = 0; r < 16; ++r) s[r] = e[r];
    }
    if (!kEarly && round + 1 < rounds) fetch(tile + kGroups, page_next);
    if (busy) {
#pragma unroll
      for (int g = 0; g < 2; ++g) {
        float e[8];
#pragma unroll
        for (int r = 0; r < 8; ++r) e[r] = s[8 * g + r];
        Op p[3];
        split::split3_even(e, p);
        Op v[2][3];
        auto read_values = [&](int c) {
#pragma unroll
          for (int part = 0; part < 3; ++part) {
            const int at = part * kValuePart + 16 * g * kValueRow + 64 * c;
            v[c & 1][part].h[0] = lds_transposed(v_lane, at);
            v[c & 1][part].h[1] = lds_transposed(v_lane, at + 8 * kValueRow);
          }
        };
        read_values(0);
#pragma unroll
        for (int c = 0; c < kColTiles; ++c) {
          if (c + 1 < kColTiles) read_values(c + 1);
          o[c] = split::mfma6(v[c & 1], p, o[c]);
          if (DP > 64) asm volatile("" ::: "memory");
        }
      }
    }
    __syncthreads();
    if (round + 1 < rounds) stage();
    __syncthreads();
  }

  l += __shfl_xor(l, 32);
  clear_unseen(o, l);
  if (kGroups == 2 && !join_groups<DP>(*reinterpret_cast<Part<DP> *>(all_lds), group, wave, o, m, l)) return;
  finish<false, DP>(a, unit.splits == 1, blockIdx.x, mine, wave, out_row, o, m, l);
}

// Joins the parts of a unit, 32 of its columns a workgroup.
template <bool kBf16, int DP>
__global__ __launch_bounds__(kThreads) void prefill_join_kernel(const PrefillArgs a) {
  constexpr int kAbreast = 4;
  const int slot = static_cast<int>(blockIdx.x) / (DP / 32), cut = static_cast<int>(blockIdx.x) - slot * (DP / 32), hk = slot % a.d.Hk;
  const Record unit = a.record[slot];
  if (unit.splits == 0) return;
  const int lane = threadIdx.x & 63, wave = threadIdx.x / 64, local = 32 * wave + (lane & 31), h = lane / 32;
  float top = kNone, sum = 0.f;
  f32x4 o[4] = {};
  for (int split0 = 0; split0 < unit.splits; split0 += kAbreast) {
    float m[kAbreast], l[kAbreast];
    f32x4 q[kAbreast][4];
#pragma unroll
    for (int s = 0; s < kAbreast; ++s) {
      const int at = slot + (split0 + s) * a.d.Hk;
      m[s] = kNone;
      l[s] = 0.f;
#pragma unroll
      for (int i = 0; i < 4; ++i) q[s][i] = f32x4{0.f, 0.f, 0.f, 0.f};
      if (split0 + s < unit.splits && at < a.parts) {  // (boundaries that make sequences overlap could have more than there is room for)
        const Part<DP> &part = static_cast<const Part<DP> *>(a.part)[at];
        m[s] = part.m[wave][lane];
        l[s] = part.l[wave][lane];
#pragma unroll
        for (int i = 0; i < 4; ++i) q[s][i] = part.o[wave][4 * cut + i][lane];
      }
    }
    float next = top;
#pragma unroll
    for (int s = 0; s < kAbreast; ++s) next = fmaxf(next, m[s]);
    const float keep = __builtin_amdgcn_exp2f(top - next);
    top = next;
    sum *= keep;
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int r = 0; r < 4; ++r) o[i][r] *= keep;
#pragma unroll
    for (int s = 0; s < kAbreast; ++s) {
      const float f = __builtin_amdgcn_exp2f(m[s] - next);
      sum = fmaf(l[s], f, sum);
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int r = 0; r < 4; ++r) o[i][r] = fmaf(q[s][i][r], f, o[i][r]);
    }
  }
  if (local >= unit.rows) return;
  const float inv = sum == 0.f ? 0.f : 1.f / sum;
  const int row = unit.first_row + local, token = quotient(row, a.d.G, a.inv_group);
  const int64_t out_row = static_cast<int64_t>(unit.begin + token) * a.d.H + hk * a.d.G + (row - token * a.d.G);
#pragma unroll
  for (int i = 0; i < 4; ++i) write_row<kBf16>(a, out_row, piece_column(4 * cut + i, h), o[i], inv);
}

struct Plan {
  int units, groups;
  int64_t tiles;  // at most, of a unit
  bool shared;
};
// bf16: two groups of waves share a unit where that leaves every CU a workgroup or few more: 2048 tokens, 32 heads over 8 of 128, 520
// units: 52 us, with a group each 56; 4096 tokens, 1032 units: 170 and 155.  Units of few tiles are not worth it: four times 512
// tokens, 8 tiles: 31 and 25; 1024 tokens, 16 tiles: 24 and 27; but where there is a CU for each, once 512 tokens: 17.4 and 18.3, 200
// tokens, 4 tiles: 12.8 and 11.6.
//
// A unit's tiles may be shared by several workgroups where that could shorten the longest row of units a CU works on by more than
// the parts' way through memory and the second launch take.  The host knows the rows of all sequences together, not of each, and
// the most tokens that the page table holds; by how many, the device finds (find_unit).
Plan plan_of(const AttnDims &d) {
  Plan p;
  const int64_t rows = static_cast<int64_t>(d.T) * d.G;
  p.units = static_cast<int>(rows / kUnitRows + d.B);
  const int64_t all = static_cast<int64_t>(p.units) * d.Hk;
  const int64_t most_seen = d.window > 0 ? std::min<int64_t>(d.capacity(), static_cast<int64_t>(d.window) + kUnitRows / d.G) : d.capacity();
  const int64_t tiles = p.tiles = (most_seen + tokens_of_tile(d.bf16) - 1) / tokens_of_tile(d.bf16);
  p.groups = d.bf16 && d.D <= 128 && all < kManyUnits && tiles >= (all <= kWorkgroups ? kFewTiles : kManyTiles) ? 2 : 1;
  p.shared = false;
  if (all >= kManyUnits) return p;
  // in us: a tile on a CU, a part written and read
  const double tile = (d.bf16 ? 1.0 : 2.0) * d.D / 128, part = 0.04 * d.D / 128, launch = 5.0;
  const double units = (std::ceil(static_cast<double>(rows) / kUnitRows) + 0.5 * (d.B - 1)) * d.Hk;
  // whole prompts, whose units see from no tile to all: the longest first fills the CUs evenly; pieces behind a long cache see much
  // the same each, and the last CU to begin one decides
  const bool prompts = most_seen <= 2 * static_cast<int64_t>(d.T / d.B);
  double whole = 0.0;
  for (int s = 1; s == 1 || (s <= kMostSplits && (s - 1) * least_tiles(d) < tiles); ++s) {
    const double longest = static_cast<double>(tiles) / s;
    const double row = prompts ? std::max(longest, units * tiles / 2 / kWorkgroups) + longest / 4 : std::ceil(units * s / kWorkgroups) * longest;
    const double cost = row * tile + (s > 1 ? launch + part * units * s : 0.0);
    if (s == 1) whole = cost;
    else p.shared |= cost < whole;
  }
  return p;
}

template <bool kBf16, int DP>
hipError_t launch(const PrefillArgs &a, hipStream_t stream) {
  const dim3 grid(static_cast<unsigned>(a.units) * a.d.Hk + (a.splits > 1 ? kMostParts : 0));
  constexpr int kTwo = DP <= 128 ? 2 : 1;  // (heads of 256 values leave registers for one wave a SIMD)
  const bool two = kTwo == 2 && a.groups == 2;
  const dim3 threads(two ? 2 * kThreads : kThreads);
  if constexpr (!kBf16) {
    hipLaunchKernelGGL(prefill_f32_kernel<DP>, grid, dim3(kThreads * f32_groups(DP)), 0, stream, a);
  } else if (a.d.D == DP) {
    if (two)
      hipLaunchKernelGGL((prefill_bf16_kernel<DP, true, kTwo>), grid, threads, 0, stream, a);
    else
      hipLaunchKernelGGL((prefill_bf16_kernel<DP, true, 1>), grid, threads, 0, stream, a);
  } else {
    if (two)
      hipLaunchKernelGGL((prefill_bf16_kernel<DP, false, kTwo>), grid, threads, 0, stream, a);
    else
      hipLaunchKernelGGL((prefill_bf16_kernel<DP, false, 1>), grid, threads, 0, stream, a);
  }
  if (const hipError_t e = hipGetLastError(); e != hipSuccess || a.splits == 1) return e;
  hipLaunchKernelGGL((prefill_join_kernel<kBf16, DP>), dim3(grid.x * (DP / 32)), dim3(kThreads), 0, stream, a);
  return hipGetLastError();
}
template <bool kBf16>
hipError_t launch(const PrefillArgs &a, hipStream_t stream) {
  return a.d.D <= 64 ? launch<kBf16, 64>(a, stream) : a.d.D <= 128 ? launch<kBf16, 128>(a, stream) : launch<kBf16, 256>(a, stream);
}

size_t part_bytes(const AttnDims &d) { return d.D <= 64 ? sizeof(Part<64>) : d.D <= 128 ? sizeof(Part<128>) : sizeof(Part<256>); }

}  // namespace

bool attn_prefill_fits(const AttnDims &d) { return static_cast<int64_t>(plan_of(d).units) * d.Hk <= kMostWorkgroups256; }

namespace {

size_t bytes_of(const AttnDims &d, int64_t units) {
  return (static_cast<size_t>(units + kMostParts) * (part_bytes(d) + sizeof(Record)) + 255) / 256 * 256;
}

}  // namespace

size_t attn_prefill_used_bytes(const AttnDims &d) {
  const Plan p = plan_of(d);
  return p.shared ? bytes_of(d, static_cast<int64_t>(p.units) * d.Hk) : 256;
}
size_t attn_prefill_workspace_bytes(const AttnDims &d) {
  const Plan p = plan_of(d);
  if (p.tiles <= least_tiles(d)) return 256;  // (no unit has two splits' tiles)
  return bytes_of(d, std::min<int64_t>(static_cast<int64_t>(p.units) * d.Hk, kManyUnits - 1));
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
  a.d = d;
  a.inv_group = inverse_of(d.G);
  a.units = p.units;
  a.splits = p.shared ? kMostSplits : 1;
  a.least = least_tiles(d);
  a.parts = p.shared ? p.units * d.Hk + kMostParts : 0;
  a.part = workspace;
  a.record = reinterpret_cast<Record *>(static_cast<char *>(workspace) + a.parts * part_bytes(d));
  a.groups = p.groups;
  a.scale_log2 = scale * 1.44269504f;
  return d.bf16 ? launch<true>(a, stream) : launch<false>(a, stream);
}

}  // namespace ssd
