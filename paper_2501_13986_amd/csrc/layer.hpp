// Host side of the gated feed-forward block (gated_f32.hip, gated_f64.hip): arguments are checked by the entry points in
// api_layer.cpp.
#pragma once

#include <hip/hip_runtime_api.h>

#include <cstddef>
#include <cstdint>

namespace cgtp {

struct GatedArgs {
  const void *x, *Wg, *Wu, *bg, *bu, *gout;
  void *out, *gx, *gWg, *gWu, *gbg, *gbu;
  int64_t rows, d_in, d_out, ld_x, ld_out, ld_gout, ld_gx;
  int act;
};

// Everything is enqueued on `st`; nothing is allocated and nothing synchronises.  cus: compute units of the current device, at most
// 256.  The workspace does not depend on them.
hipError_t gated_forward_f32(const GatedArgs& a, int cus, hipStream_t st);
hipError_t gated_forward_f64(const GatedArgs& a, int cus, hipStream_t st);
size_t gated_workspace_bytes_f32(int64_t rows, int64_t d_in, int64_t d_out);
size_t gated_workspace_bytes_f64(int64_t rows, int64_t d_in, int64_t d_out);
hipError_t gated_backward_f32(const GatedArgs& a, int cus, void* workspace, hipStream_t st);
hipError_t gated_backward_f64(const GatedArgs& a, int cus, void* workspace, hipStream_t st);

}  // namespace cgtp
