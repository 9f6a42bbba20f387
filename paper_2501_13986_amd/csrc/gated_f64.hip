// Gated feed-forward block, double precision.
#include "gated_kernels.hpp"

namespace cgtp {

hipError_t gated_forward_f64(const GatedArgs& a, int cus, hipStream_t st) { return forward<double>(a, cus, st); }
size_t gated_workspace_bytes_f64(int64_t rows, int64_t d_in, int64_t d_out) { return workspace_bytes<double>(rows, d_in, d_out); }
hipError_t gated_backward_f64(const GatedArgs& a, int cus, void* ws, hipStream_t st) { return backward<double>(a, cus, (char*)ws, st); }

}  // namespace cgtp
