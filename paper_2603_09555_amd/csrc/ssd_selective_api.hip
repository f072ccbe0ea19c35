// C ABI of the selective scan (declared in include/ssd.h): host-side validation and dispatch.  Every check runs before the
// first HIP call, so an invalid call enqueues nothing.
#include "ssd_selective.hpp"

namespace {

using ssd::SelectiveDims;

bool aligned(const void *p, uintptr_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }

ssd_status make_dims(const ssd_selective_shape *s, bool packed, SelectiveDims *out) {
  if (!s) return SSD_ERR_NULL;
  if ((s->io_dtype != SSD_F32 && s->io_dtype != SSD_BF16) || (s->dt_dtype != SSD_F32 && s->dt_dtype != s->io_dtype)) return SSD_ERR_DTYPE;
  if (s->batch < 1 || (packed && s->tokens < 1) || s->channels < 1 || s->dstate < 1) return SSD_ERR_SHAPE;
  if (s->dstate > ssd::kMostSelectiveStates) return SSD_ERR_UNSUPPORTED;
  SelectiveDims d = {};
  d.B = s->batch;
  d.T = packed ? s->tokens : s->batch;
  d.C = s->channels;
  d.N = s->dstate;
  d.bf16 = s->io_dtype == SSD_BF16;
  d.dt_bf16 = s->dt_dtype == SSD_BF16;
  // lanes count channels, and the rest is addressed with head-room
  if (d.C > (1 << 22) || d.T > (1 << 30) || d.B > (1 << 30) || static_cast<long double>(d.B) * d.C * d.N > 1.0e15L) return SSD_ERR_SHAPE;
  *out = d;
  return SSD_OK;
}
ssd_status prefill_dims(const ssd_selective_shape *s, SelectiveDims *d) {
  const ssd_status st = make_dims(s, true, d);
  return st == SSD_OK && !ssd::selective_prefill_fits(*d) ? SSD_ERR_SHAPE : st;
}

// What both calls check of their tensors and strides.
ssd_status selective_args(SelectiveDims *d, const ssd_dt_transform *dtx, const void *x, const void *dt, const float *A, const void *B,
                          int64_t B_stride, const void *C, int64_t C_stride, const float *D, const void *z, int64_t z_stride, const void *y) {
  if (dtx) {
    if (dtx->dt_max > 0.f && !(dtx->dt_min <= dtx->dt_max)) return SSD_ERR_SHAPE;
    d->dtx = {dtx->dt_bias, dtx->dt_softplus != 0, dtx->dt_min, dtx->dt_max};
  }
  if (B_stride < d->N || C_stride < d->N || (z && z_stride < d->C)) return SSD_ERR_SHAPE;
  for (const int64_t stride : {B_stride, C_stride, z ? z_stride : 0})
    if (stride > (1 << 24)) return SSD_ERR_UNSUPPORTED;  // (sixteen rows are addressed with 31 bits)
  if (!x || !dt || !A || !B || !C || !y) return SSD_ERR_NULL;
  const uintptr_t element = d->bf16 ? 2 : 4;
  for (const void *p : {B, C, z})
    if (!aligned(p, element)) return SSD_ERR_ALIGN;
  for (const void *p : {x, dt, static_cast<const void *>(A), static_cast<const void *>(D), static_cast<const void *>(d->dtx.bias), y})
    if (!aligned(p, 16)) return SSD_ERR_ALIGN;
  return SSD_OK;
}

}  // namespace

extern "C" {

size_t ssd_selective_prefill_workspace_bytes(const ssd_selective_shape *shape) {
  SelectiveDims d;
  return prefill_dims(shape, &d) == SSD_OK ? ssd::selective_prefill_workspace_bytes(d) : 0;
}

ssd_status ssd_selective_prefill(const ssd_selective_shape *shape, const ssd_dt_transform *dt_transform, const int32_t *cu_seqlens,
                                 const void *x, const void *dt, const float *A, const void *B, int64_t B_stride, const void *C,
                                 int64_t C_stride, const float *D, const void *z, int64_t z_stride, const float *h0, void *y,
                                 float *final_state, void *workspace, size_t workspace_bytes, void *hip_stream) {
  SelectiveDims d;
  if (const ssd_status st = prefill_dims(shape, &d); st != SSD_OK) return st;
  if (const ssd_status st = selective_args(&d, dt_transform, x, dt, A, B, B_stride, C, C_stride, D, z, z_stride, y); st != SSD_OK) return st;
  if (!cu_seqlens || !final_state) return SSD_ERR_NULL;
  if (!aligned(cu_seqlens, 4) || !aligned(h0, 16) || !aligned(final_state, 16)) return SSD_ERR_ALIGN;
  if (!workspace || !aligned(workspace, 256) || workspace_bytes < ssd::selective_prefill_workspace_bytes(d)) return SSD_ERR_WORKSPACE;
  const ssd::SelectiveArgs a = {x, dt, B, C, z, A, D, B_stride, C_stride, z_stride, y};
  return ssd::launch_selective_prefill(d, a, cu_seqlens, h0, final_state, workspace, static_cast<hipStream_t>(hip_stream)) == hipSuccess ? SSD_OK
                                                                                                                                      : SSD_ERR_HIP;
}

ssd_status ssd_selective_step(const ssd_selective_shape *shape, const ssd_dt_transform *dt_transform, float *state, const void *x, const void *dt,
                              const float *A, const void *B, int64_t B_stride, const void *C, int64_t C_stride, const float *D, const void *z,
                              int64_t z_stride, void *y, void *hip_stream) {
  SelectiveDims d;
  if (const ssd_status st = make_dims(shape, false, &d); st != SSD_OK) return st;
  if (!ssd::selective_step_fits(d)) return SSD_ERR_SHAPE;
  if (const ssd_status st = selective_args(&d, dt_transform, x, dt, A, B, B_stride, C, C_stride, D, z, z_stride, y); st != SSD_OK) return st;
  if (!state) return SSD_ERR_NULL;
  if (!aligned(state, 16)) return SSD_ERR_ALIGN;
  const ssd::SelectiveArgs a = {x, dt, B, C, z, A, D, B_stride, C_stride, z_stride, y};
  return ssd::launch_selective_step(d, a, state, static_cast<hipStream_t>(hip_stream)) == hipSuccess ? SSD_OK : SSD_ERR_HIP;
}

}  // extern "C"
