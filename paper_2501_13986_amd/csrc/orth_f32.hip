// Orthogonalised updates, single precision.
#include "orth_kernels.hpp"

namespace cgtp {

size_t orth_workspace_bytes_f32(int64_t batch, int64_t m, int64_t n) { return workspace_bytes<float>(batch, m, n); }
hipError_t orth_f32(const OrthArgs& a, const double* coefficients, int steps, void* ws, hipStream_t st) { return orthogonalise<float>(a, coefficients, steps, (char*)ws, st); }

}  // namespace cgtp
