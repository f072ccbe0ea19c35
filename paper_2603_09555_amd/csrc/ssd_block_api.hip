// C ABI of the operators of a hybrid stack's other layers (declared in include/ssd.h): host-side validation and dispatch.
// Every check runs before the first HIP call, so an invalid call enqueues nothing.
#include "ssd_block.hpp"

namespace {

using ssd::AttnDims;

bool aligned16(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }
bool aligned4(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 3u) == 0; }
bool is_dtype(int32_t t) { return t == SSD_F32 || t == SSD_BF16; }

// Shared checks of the two norms.
ssd_status norm_shape(int64_t rows, int32_t width, int32_t groups, int32_t io_dtype, float eps) {
  if (!is_dtype(io_dtype)) return SSD_ERR_DTYPE;
  if (rows < 1 || width < 1 || groups < 1 || width % groups != 0 || !(eps >= 0.f)) return SSD_ERR_SHAPE;
  if (static_cast<long double>(rows) * groups > 2147483647.0L || width > (1 << 30)) return SSD_ERR_SHAPE;
  if (static_cast<long double>(rows) * width > 1.0e15L) return SSD_ERR_SHAPE;
  return SSD_OK;
}

ssd_status make_dims(const ssd_attn_shape *s, bool packed, AttnDims *out) {
  if (!s) return SSD_ERR_NULL;
  if (!is_dtype(s->io_dtype)) return SSD_ERR_DTYPE;
  if (s->batch < 1 || (packed && s->tokens < 1) || s->nheads < 1 || s->nkvheads < 1 || s->headdim < 1 || s->npages < 1 ||
      s->page_size < 1 || s->max_pages < 1 || s->window < 0)
    return SSD_ERR_SHAPE;
  if (s->nheads % s->nkvheads != 0) return SSD_ERR_SHAPE;
  if (s->headdim > 256 || s->headdim % 8 != 0 || s->page_size > 65536 || (s->page_size & (s->page_size - 1)) != 0 ||
      s->nheads > 65535)
    return SSD_ERR_UNSUPPORTED;
  AttnDims d = {};
  d.B = s->batch;
  d.T = packed ? s->tokens : s->batch;
  d.H = s->nheads;
  d.Hk = s->nkvheads;
  d.D = s->headdim;
  d.G = d.H / d.Hk;
  d.npages = s->npages;
  while ((1 << d.lg_page) < s->page_size) ++d.lg_page;
  d.max_pages = s->max_pages;
  d.bf16 = s->io_dtype == SSD_BF16;
  // positions fit 30 bits; tensors are addressable with head-room
  if (static_cast<long double>(d.max_pages) * s->page_size > 1073741824.0L) return SSD_ERR_SHAPE;
  // a window as wide as a row of the page table is no limit, and positions minus smaller ones fit 32 bits
  d.window = s->window < d.capacity() ? s->window : 0;
  if (static_cast<long double>(d.npages) * d.Hk * s->page_size * d.D > 1.0e15L || d.T > (1 << 30) || d.B > (1 << 30) ||
      static_cast<long double>(d.T) * d.H > 2147483647.0L || static_cast<long double>(d.B) * d.H > 2147483647.0L)
    return SSD_ERR_SHAPE;
  // a page of the cache is addressed with 32 bits
  if (static_cast<long double>(d.Hk) * s->page_size * d.D * (d.bf16 ? 2 : 4) > 2147483647.0L) return SSD_ERR_UNSUPPORTED;
  *out = d;
  return SSD_OK;
}

ssd_status step_dims(const ssd_attn_shape *s, AttnDims *d) {
  const ssd_status st = make_dims(s, false, d);
  return st == SSD_OK && !ssd::attn_step_fits(*d) ? SSD_ERR_SHAPE : st;
}
ssd_status prefill_dims(const ssd_attn_shape *s, AttnDims *d) {
  const ssd_status st = make_dims(s, true, d);
  return st == SSD_OK && !ssd::attn_prefill_fits(*d) ? SSD_ERR_SHAPE : st;
}

// The device arrays and the caches, of either attention call.
ssd_status attn_pointers(const int32_t *seq_lens, const int32_t *page_table, const void *q, const void *k_cache,
                         const void *v_cache, const void *y) {
  if (!seq_lens || !page_table || !q || !k_cache || !v_cache || !y) return SSD_ERR_NULL;
  if (!aligned4(seq_lens) || !aligned4(page_table) || !aligned16(q) || !aligned16(k_cache) || !aligned16(v_cache) ||
      !aligned16(y))
    return SSD_ERR_ALIGN;
  return SSD_OK;
}

// A scale of the logits: positive and finite.
bool scale_ok(float scale) { return scale > 0.f && scale <= 1.0e30f; }

// Whether `bytes` at `out` reach into one of `count` rows of `row` bytes, `stride` apart.
bool reaches(const void *out, int64_t bytes, const void *rows, int64_t stride, int64_t row, int64_t count) {
  const uintptr_t o = reinterpret_cast<uintptr_t>(out), first = reinterpret_cast<uintptr_t>(rows);
  if (o + bytes <= first || o >= first + (count - 1) * stride + row) return false;
  if (o < first) return true;
  const int64_t at = static_cast<int64_t>((o - first) % static_cast<uintptr_t>(stride));  // (behind the row, up to the next one: a gap)
  return at < row || at + bytes > stride;
}

bool workspace_ok(const void *workspace, size_t given, size_t need) {
  return workspace && given >= need && (reinterpret_cast<uintptr_t>(workspace) & 255u) == 0;
}

ssd_status status_of(hipError_t e) { return e == hipSuccess ? SSD_OK : SSD_ERR_HIP; }

}  // namespace

extern "C" {

ssd_status ssd_norm_gated(int64_t rows, int32_t width, int32_t groups, int32_t io_dtype, const void *y, const void *z,
                          int64_t z_stride, const float *weight, float eps, int32_t norm_first, void *out, void *hip_stream) {
  if (const ssd_status st = norm_shape(rows, width, groups, io_dtype, eps); st != SSD_OK) return st;
  if (z_stride < width || static_cast<long double>(z_stride) * rows > 1.0e15L || (norm_first != 0 && norm_first != 1))
    return SSD_ERR_SHAPE;
  if (!y || !z || !weight || !out) return SSD_ERR_NULL;
  const uintptr_t element = io_dtype == SSD_BF16 ? 2 : 4;
  if (!aligned16(y) || !aligned16(weight) || !aligned16(out) || reinterpret_cast<uintptr_t>(z) % element != 0) return SSD_ERR_ALIGN;
  return status_of(ssd::launch_norm_gated(rows, width, groups, io_dtype == SSD_BF16, y, z, z_stride, weight, eps, norm_first != 0,
                                          out, static_cast<hipStream_t>(hip_stream)));
}

ssd_status ssd_norm_residual(int64_t rows, int32_t width, int32_t io_dtype, int32_t residual_dtype, const void *x,
                             const void *residual, float scale, const float *weight, float eps, void *out, void *residual_out,
                             void *hip_stream) {
  if (const ssd_status st = norm_shape(rows, width, 1, io_dtype, eps); st != SSD_OK) return st;
  if (residual_dtype != SSD_F32 && residual_dtype != io_dtype) return SSD_ERR_DTYPE;
  if (!x || !weight || !out || !residual_out) return SSD_ERR_NULL;
  if (!aligned16(x) || !aligned16(weight) || !aligned16(out) || !aligned16(residual_out) || (residual && !aligned16(residual)))
    return SSD_ERR_ALIGN;
  return status_of(ssd::launch_norm_residual(rows, width, io_dtype == SSD_BF16, residual_dtype == SSD_BF16, x, residual, scale,
                                             weight, eps, out, residual_out, static_cast<hipStream_t>(hip_stream)));
}

ssd_status ssd_attn_append(const ssd_attn_shape *shape, const ssd_rope *rope, const int32_t *cu_seqlens, const int32_t *seq_lens,
                           const int32_t *page_table, const void *q, int64_t q_stride, const void *k, int64_t k_stride,
                           const void *v, int64_t v_stride, void *q_out, void *k_cache, void *v_cache, void *hip_stream) {
  AttnDims d;
  if (const ssd_status st = make_dims(shape, cu_seqlens != nullptr, &d); st != SSD_OK) return st;
  if (!ssd::attn_append_fits(d, q != nullptr)) return SSD_ERR_SHAPE;
  if (!rope || !seq_lens || !page_table || !k || !v || !k_cache || !v_cache || (q == nullptr) != (q_out == nullptr))
    return SSD_ERR_NULL;
  if (rope->rotary < 0 || rope->rotary % 2 != 0 || rope->rotary > d.D || (rope->interleaved != 0 && rope->interleaved != 1))
    return SSD_ERR_SHAPE;
  if (rope->rotary > 0) {
    if (!rope->cos || !rope->sin) return SSD_ERR_NULL;
    if (!aligned16(rope->cos) || !aligned16(rope->sin)) return SSD_ERR_ALIGN;
    if (rope->positions < d.capacity()) return SSD_ERR_SHAPE;
  }
  const int64_t piece = d.bf16 ? 8 : 4;
  const int64_t strides[3] = {q ? q_stride : static_cast<int64_t>(d.H) * d.D, k_stride, v_stride};
  for (int i = 0; i < 3; ++i) {
    const int64_t row = static_cast<int64_t>(i == 0 ? d.H : d.Hk) * d.D;
    if (strides[i] < row || static_cast<long double>(strides[i]) * d.T > 1.0e15L) return SSD_ERR_SHAPE;
    if (strides[i] % piece != 0) return SSD_ERR_ALIGN;
  }
  if (!aligned4(seq_lens) || !aligned4(page_table) || !aligned4(cu_seqlens) ||
      !aligned16(q) || !aligned16(k) || !aligned16(v) || !aligned16(q_out) || !aligned16(k_cache) || !aligned16(v_cache))
    return SSD_ERR_ALIGN;
  if (q) {  // a thread that rotates reads what its neighbour writes
    const int64_t size = d.bf16 ? 2 : 4, head = d.D * size, out = static_cast<int64_t>(d.T) * d.H * head;
    const void *const from[3] = {q, k, v};
    for (int i = 0; i < 3; ++i)
      if (reaches(q_out, out, from[i], strides[i] * size, (i == 0 ? d.H : d.Hk) * head, d.T)) return SSD_ERR_UNSUPPORTED;
  }
  const ssd::Rope r = {rope->cos, rope->sin, rope->rotary / 2, rope->interleaved};
  return status_of(ssd::launch_attn_append(d, r, cu_seqlens, seq_lens, page_table, q, strides[0], k, k_stride, v, v_stride, q_out,
                                           k_cache, v_cache, static_cast<hipStream_t>(hip_stream)));
}

size_t ssd_attn_step_workspace_bytes(const ssd_attn_shape *shape) {
  AttnDims d;
  return step_dims(shape, &d) == SSD_OK ? ssd::attn_step_workspace_bytes(d) : 0;
}

ssd_status ssd_attn_step(const ssd_attn_shape *shape, const int32_t *seq_lens, const int32_t *page_table, const void *q,
                         const void *k_cache, const void *v_cache, float scale, void *y, void *workspace, size_t workspace_bytes,
                         void *hip_stream) {
  AttnDims d;
  if (const ssd_status st = step_dims(shape, &d); st != SSD_OK) return st;
  if (!scale_ok(scale)) return SSD_ERR_SHAPE;
  if (const ssd_status st = attn_pointers(seq_lens, page_table, q, k_cache, v_cache, y); st != SSD_OK) return st;
  if (!workspace_ok(workspace, workspace_bytes, ssd::attn_step_used_bytes(d))) return SSD_ERR_WORKSPACE;
  return status_of(ssd::launch_attn_step(d, seq_lens, page_table, q, k_cache, v_cache, scale, y, workspace,
                                         static_cast<hipStream_t>(hip_stream)));
}

size_t ssd_attn_prefill_workspace_bytes(const ssd_attn_shape *shape) {
  AttnDims d;
  return prefill_dims(shape, &d) == SSD_OK ? ssd::attn_prefill_workspace_bytes(d) : 0;
}

ssd_status ssd_attn_prefill(const ssd_attn_shape *shape, const int32_t *cu_seqlens, const int32_t *seq_lens,
                            const int32_t *page_table, const void *q, const void *k_cache, const void *v_cache, float scale,
                            void *y, void *workspace, size_t workspace_bytes, void *hip_stream) {
  AttnDims d;
  if (const ssd_status st = prefill_dims(shape, &d); st != SSD_OK) return st;
  if (!scale_ok(scale)) return SSD_ERR_SHAPE;
  if (!cu_seqlens) return SSD_ERR_NULL;
  if (const ssd_status st = attn_pointers(seq_lens, page_table, q, k_cache, v_cache, y); st != SSD_OK) return st;
  if (!aligned4(cu_seqlens)) return SSD_ERR_ALIGN;
  if (!workspace_ok(workspace, workspace_bytes, ssd::attn_prefill_used_bytes(d))) return SSD_ERR_WORKSPACE;
  return status_of(ssd::launch_attn_prefill(d, cu_seqlens, seq_lens, page_table, q, k_cache, v_cache, scale, y, workspace,
                                            static_cast<hipStream_t>(hip_stream)));
}

}  // extern "C"
