// Orthogonalised updates, double precision.
#include "orth_kernels.hpp"

namespace cgtp {

size_t orth_workspace_bytes_f64(int64_t batch, int64_t m, int64_t n) { return workspace_bytes<double>(batch, m, n); }
hipError_t orth_f64(const OrthArgs& a, const double* coefficients, int steps, void* ws, hipStream_t st) { return orthogonalise<double>(a, coefficients, steps, (char*)ws, st); }

}  // namespace cgtp
