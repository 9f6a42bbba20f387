// Host side of the products by kind of row (grouped_f32.hip, grouped_f64.hip): arguments are checked by the entry points in api_products.cpp.
#pragma once

#include <hip/hip_runtime_api.h>

#include <cstddef>
#include <cstdint>

namespace cgtp {

struct GroupedArgs {
  const void *x, *W, *b, *gout;
  void *out, *gx, *gW, *gb;
  int64_t rows, d_in, d_out, comps, groups, ld_x, ld_out, ld_gout, ld_gx;
  const int64_t *ptr, *perm;
};

// Everything is enqueued on `st`; nothing is allocated and nothing synchronises.
hipError_t grouped_forward_f32(const GroupedArgs& a, hipStream_t st);
hipError_t grouped_forward_f64(const GroupedArgs& a, hipStream_t st);
size_t grouped_workspace_bytes_f32(int64_t rows, int64_t d_in, int64_t d_out, int64_t comps);
size_t grouped_workspace_bytes_f64(int64_t rows, int64_t d_in, int64_t d_out, int64_t comps);
hipError_t grouped_backward_f32(const GroupedArgs& a, void* workspace, hipStream_t st);
hipError_t grouped_backward_f64(const GroupedArgs& a, void* workspace, hipStream_t st);

}  // namespace cgtp
