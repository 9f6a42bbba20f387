// Host side of the layer operators (gated.hip, norm.cpp): arguments are checked by the entry points in api_layer.cpp.
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
  bool f64;
};
hipError_t gated_forward(const GatedArgs& a, hipStream_t st);
size_t gated_workspace_bytes(int64_t rows, int64_t d_in, int64_t d_out, bool f64);
hipError_t gated_backward(const GatedArgs& a, void* workspace, hipStream_t st);

}  // namespace cgtp
