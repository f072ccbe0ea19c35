// Device code shared by the operators on a paged key-value cache: where a token and its page are.
#pragma once

#include <type_traits>

#include "ssd_block.hpp"

namespace ssd {

// A sequence's length as the kernels use it.
__device__ __forceinline__ int cut_length(const AttnDims &d, int len) { return min(max(len, 0), d.capacity()); }

struct Token {
  int seq, pos;  // pos < 0: in front of its sequence's beginning
  bool found;    // in a sequence
};

// The sequence and position of a packed new token (cu == nullptr: one for each sequence).  All lanes of a wave ask for the
// same token: 64 boundaries are compared at a time.
__device__ __forceinline__ Token find_token(const AttnDims &d, const int32_t *cu, const int32_t *lens, int token) {
  Token t = {token, -1, cu == nullptr};
  int end = token + 1;
  if (cu != nullptr) {
    int last = -1;  // the last sequence that begins at or in front of the token (and, being last, is not empty)
    for (int b0 = 0; b0 < d.B; b0 += 64) {
      const int b = b0 + (threadIdx.x & 63);
      const uint64_t m = __ballot(b < d.B && cu[b] <= token);
      if (m != 0) last = b0 + 63 - __builtin_clzll(m);
    }
    if (last < 0) return t;
    t.seq = last;
    end = min(cu[last + 1], d.T);
    if (token >= end) return t;
    t.found = true;
  }
  t.pos = cut_length(d, lens[t.seq]) - (end - token);
  return t;
}

// The cache row (of headdim values) of a sequence's token for a key head, or -1 if its page is not in the cache.
__device__ __forceinline__ int64_t slot_of(const AttnDims &d, const int32_t *table, int seq, int pos, int head) {
  const int page = table[static_cast<int64_t>(seq) * d.max_pages + (pos >> d.lg_page)];
  if (static_cast<unsigned>(page) >= static_cast<unsigned>(d.npages)) return -1;
  return ((static_cast<int64_t>(page) * d.Hk + head) << d.lg_page) + (pos & ((1 << d.lg_page) - 1));
}

}  // namespace ssd
