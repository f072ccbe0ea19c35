// Device code shared by the operators on a paged key-value cache: where a token and its page are.
#pragma once

#include <type_traits>

#include "ssd_block.hpp"

namespace ssd {

struct Token {
  int seq, pos;  // pos < 0: in no sequence, or without a place in it (in front of its beginning, behind its row of the table)
};

// The sequence and position of a packed new token (cu == nullptr: one for each sequence).
__device__ __forceinline__ Token find_token(const AttnDims &d, const int32_t *cu, const int32_t *lens, int token) {
  Token t = {token, -1};
  int end = token + 1;
  if (cu != nullptr) {
    int last = 0, behind = d.B;  // the last sequence that begins at or in front of the token (and, being last, is not empty)
    while (behind - last > 1) {
      const int b = (last + behind) / 2;
      if (cu[b] <= token) last = b;
      else behind = b;
    }
    end = min(cu[last + 1], d.T);
    if (cu[last] > token || token >= end) return t;
    t.seq = last;
  }
  t.pos = max(lens[t.seq], 0) - (end - token);
  if (t.pos >= d.capacity()) t.pos = -1;
  return t;
}

// The cache row (of headdim values) of a sequence's token for a key head, or -1 if its page is not in the cache.
__device__ __forceinline__ int64_t slot_of(const AttnDims &d, const int32_t *table, int seq, int pos, int head) {
  const int page = table[static_cast<int64_t>(seq) * d.max_pages + (pos >> d.lg_page)];
  if (static_cast<unsigned>(page) >= static_cast<unsigned>(d.npages)) return -1;
  return ((static_cast<int64_t>(page) * d.Hk + head) << d.lg_page) + (pos & ((1 << d.lg_page) - 1));
}

// Work that is dealt to workgroups in equal runs is one long list of blocks, those of each item in a row.  Prefix::at[t]: blocks of
// the items in front of thread t's share of them, [kDealers]: of all.
constexpr int kDealers = 256;  // threads of a workgroup
struct Prefix {
  int64_t at[kDealers + 1];
  int64_t wave[kDealers / 64];
};
__device__ __forceinline__ int share_of(int items) { return (items + kDealers - 1) / kDealers; }
template <typename Blocks>
__device__ __forceinline__ void count_blocks(Prefix &s, int items, const Blocks &blocks_of) {
  const int t = threadIdx.x, lane = t & 63, share = share_of(items);
  int64_t sum = 0;
  for (int64_t i = static_cast<int64_t>(t) * share; i < min(static_cast<int64_t>(t + 1) * share, static_cast<int64_t>(items)); ++i)
    sum += blocks_of(static_cast<int>(i));
#pragma unroll
  for (int k = 1; k < 64; k <<= 1) {
    const int64_t o = __shfl_up(sum, k);
    if (lane >= k) sum += o;
  }
  if (lane == 63) s.wave[t / 64] = sum;
  __syncthreads();
  for (int w = 0; w < t / 64; ++w) sum += s.wave[w];
  s.at[t + 1] = sum;
  if (t == 0) s.at[0] = 0;
  __syncthreads();
}
__device__ __forceinline__ int64_t uniform(int64_t v) {
  const uint32_t lo = __builtin_amdgcn_readfirstlane(static_cast<uint32_t>(v)), hi = __builtin_amdgcn_readfirstlane(static_cast<uint32_t>(v >> 32));
  return static_cast<int64_t>(static_cast<uint64_t>(hi) << 32 | lo);
}
// The thread whose share holds block `at`, if each item comes `times` times over.
__device__ __forceinline__ int dealer_of(const Prefix &s, int64_t at, int times) {
  int t = 0;
#pragma unroll
  for (int k = kDealers / 2; k > 0; k >>= 1)
    if (s.at[t + k] * times <= at) t += k;
  return __builtin_amdgcn_readfirstlane(t);
}

}  // namespace ssd
