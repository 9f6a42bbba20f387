// Host side of orthogonalise (orth_f32.hip, orth_f64.hip): arguments are checked by the entry point in api_products.cpp.
#pragma once

#include <hip/hip_runtime_api.h>

#include <cstddef>
#include <cstdint>

namespace cgtp {

struct OrthArgs {
  const void* g;
  void* out;
  int64_t batch, m, n, ld_g, ld_out, stride_g, stride_out;
  double eps;
};

// coefficients [steps][3], host memory.  Everything is enqueued on `st`; nothing is allocated and nothing synchronises.
size_t orth_workspace_bytes_f32(int64_t batch, int64_t m, int64_t n);
size_t orth_workspace_bytes_f64(int64_t batch, int64_t m, int64_t n);
hipError_t orth_f32(const OrthArgs& a, const double* coefficients, int steps, void* workspace, hipStream_t st);
hipError_t orth_f64(const OrthArgs& a, const double* coefficients, int steps, void* workspace, hipStream_t st);

}  // namespace cgtp
