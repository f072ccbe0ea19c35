// Causal attention of packed new tokens over a paged cache.
#include "ssd_attn_simple.hpp"

namespace ssd {

size_t attn_prefill_workspace_bytes(const AttnDims &) { return 256; }

hipError_t launch_attn_prefill(const AttnDims &d, const int32_t *cu, const int32_t *lens, const int32_t *table, const void *q,
                               const void *k_cache, const void *v_cache, float scale, void *y, void *, hipStream_t stream) {
  return launch_attn_rows(d, cu, lens, table, q, k_cache, v_cache, scale, y, stream);
}

}  // namespace ssd
