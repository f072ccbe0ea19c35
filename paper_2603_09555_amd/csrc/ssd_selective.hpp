// The selective state space scan (a decay of its own for every channel and state): what its translation units share.
#pragma once

#include "ssd_internal.hpp"

namespace ssd {

constexpr int kMostSelectiveStates = 256;

// Validated shape of a call.
struct SelectiveDims {
  int B, T, C, N;       // sequences, tokens of them all, channels, states of a channel
  bool bf16, dt_bf16;   // types of x, B, C, z, y; of dt
  DtXform dtx;
};

struct SelectiveArgs {
  const void *x, *dt, *B, *C, *z;  // z: or null
  const float *A, *D;              // D: or null
  int64_t b_stride, c_stride, z_stride;
  void *y;
};

bool selective_prefill_fits(const SelectiveDims &d);
size_t selective_prefill_workspace_bytes(const SelectiveDims &d);
hipError_t launch_selective_prefill(const SelectiveDims &d, const SelectiveArgs &a, const int32_t *cu, const float *h0, float *final_state,
                                    void *workspace, hipStream_t stream);
bool selective_step_fits(const SelectiveDims &d);
hipError_t launch_selective_step(const SelectiveDims &d, const SelectiveArgs &a, float *state, hipStream_t stream);

}  // namespace ssd
