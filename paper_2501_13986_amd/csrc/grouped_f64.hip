// Products by kind of row, double precision.
#include "grouped_kernels.hpp"

namespace cgtp {

hipError_t grouped_forward_f64(const GroupedArgs& a, hipStream_t st) { return launch_rows<double, false>(a, st); }
size_t grouped_workspace_bytes_f64(int64_t rows, int64_t d_in, int64_t d_out, int64_t comps) { return workspace_bytes<double>(rows, d_in, d_out, comps); }
hipError_t grouped_backward_f64(const GroupedArgs& a, void* ws, hipStream_t st) { return backward<double>(a, (char*)ws, st); }

}  // namespace cgtp
