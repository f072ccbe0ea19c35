// Attention of one new token of each sequence over a paged cache.
#include "ssd_attn_simple.hpp"

namespace ssd {

size_t attn_step_workspace_bytes(const AttnDims &) { return 256; }

hipError_t launch_attn_step(const AttnDims &d, const int32_t *lens, const int32_t *table, const void *q, const void *k_cache,
                            const void *v_cache, float scale, void *y, void *, hipStream_t stream) {
  return launch_attn_rows(d, nullptr, lens, table, q, k_cache, v_cache, scale, y, stream);
}

}  // namespace ssd
