// Entry points of the products by kind of row and of the orthogonalised updates.
#include <algorithm>
#include <cfloat>
#include <climits>
#include <cmath>
#include <string>

#include "csr.hpp"
#include "entry.hpp"
#include "grouped.hpp"
#include "orth.hpp"

namespace {

using cgtp::aligned;
using cgtp::bad_workspace;
using cgtp::fail;
using cgtp::workspace_serves;

constexpr int64_t kMostGroups = 1 << 24, kMostComps = 1024, kMostStride = INT32_MAX;

cgtp_status check_grouped(const cgtp::GroupedArgs& a, int32_t dtype) {
  if (dtype != CGTP_F32 && dtype != CGTP_F64) return fail(CGTP_EINVAL, "dtype must be CGTP_F32 or CGTP_F64");
  if (a.rows < 0 || a.groups < 0 || a.d_in <= 0 || a.d_out <= 0 || a.comps <= 0)
    return fail(CGTP_EINVAL, "rows and groups must not be negative, d_in, d_out and comps must be positive");
  if (a.comps > kMostComps || a.groups > kMostGroups) return fail(CGTP_EUNSUPPORTED, "comps must be at most 1024, groups at most 2^24");
  if (a.rows > INT32_MAX / a.comps) return fail(CGTP_EUNSUPPORTED, "rows times comps must be below 2^31");
  if (a.d_in > 1 << 20 || a.d_out > 1 << 20 || a.d_in > INT32_MAX / a.d_out)
    return fail(CGTP_EUNSUPPORTED, "d_in and d_out must be at most 2^20, their product below 2^31");
  for (int64_t ld : {a.ld_x, a.ld_out, a.ld_gout, a.ld_gx})
    if (ld > kMostStride) return fail(CGTP_EUNSUPPORTED, "row strides must be below 2^31");
  return CGTP_OK;
}

cgtp_status check_numbers(std::initializer_list<const void*> data, int32_t dtype) {
  for (const void* p : data)
    if (!aligned(p, dtype == CGTP_F64 ? 8 : 4)) return fail(CGTP_EINVAL, "data pointers must be aligned to their type");
  return CGTP_OK;
}

cgtp_status check_orth(int64_t batch, int64_t m, int64_t n, int32_t dtype) {
  if (dtype != CGTP_F32 && dtype != CGTP_F64) return fail(CGTP_EINVAL, "dtype must be CGTP_F32 or CGTP_F64");
  if (batch < 0 || m <= 0 || n <= 0) return fail(CGTP_EINVAL, "batch must not be negative, m and n must be positive");
  if (batch > INT32_MAX || m >= 1 << 22 || n >= 1 << 22 || m > INT32_MAX / n || batch > ((int64_t)1 << 40) / (m * n))
    return fail(CGTP_EUNSUPPORTED, "m and n must be below 2^22, batch and m n below 2^31, batch m n at most 2^40");
  return CGTP_OK;
}

}  // namespace

extern "C" {

cgtp_status grouped_forward(const void* x, const void* W, const void* b, void* out, int64_t rows, int64_t d_in, int64_t d_out,
                            int64_t comps, int64_t groups, const int64_t* ptr, const int64_t* perm, int64_t ld_x, int64_t ld_out,
                            int32_t dtype, void* hip_stream) {
  cgtp::GroupedArgs a = {};
  a.x = x; a.W = W; a.b = b; a.out = out; a.ptr = ptr; a.perm = perm;
  a.rows = rows; a.d_in = d_in; a.d_out = d_out; a.comps = comps; a.groups = groups; a.ld_x = ld_x; a.ld_out = ld_out;
  cgtp_status s = check_grouped(a, dtype);
  if (s != CGTP_OK) return s;
  if (ld_x < comps * d_in || ld_out < comps * d_out) return fail(CGTP_EINVAL, "a row stride is smaller than its row");
  if (b && comps != 1) return fail(CGTP_EINVAL, "biases are for rows of one component");
  if (rows == 0 || groups == 0) return CGTP_OK;
  if (!x || !W || !out || !ptr) return fail(CGTP_EINVAL, "NULL data pointer");
  s = check_numbers({x, W, b, out}, dtype);
  if (s != CGTP_OK) return s;
  if (!aligned(ptr, 8) || !aligned(perm, 8)) return fail(CGTP_EINVAL, "data pointers must be aligned to their type");
  HIP_TRY((dtype == CGTP_F64 ? cgtp::grouped_forward_f64 : cgtp::grouped_forward_f32)(a, (hipStream_t)hip_stream));
  return CGTP_OK;
}

size_t cgtp_grouped_workspace_bytes(int64_t rows, int64_t d_in, int64_t d_out, int64_t comps, int64_t groups, int32_t dtype) {
  cgtp::GroupedArgs a = {};
  a.rows = rows; a.d_in = d_in; a.d_out = d_out; a.comps = comps; a.groups = groups;
  if (check_grouped(a, dtype) != CGTP_OK || rows == 0 || groups == 0) return 0;
  return (dtype == CGTP_F64 ? cgtp::grouped_workspace_bytes_f64 : cgtp::grouped_workspace_bytes_f32)(rows, d_in, d_out, comps);
}

cgtp_status grouped_backward(const void* x, const void* W, const void* gout, void* gx, void* gW, void* gb, int64_t rows, int64_t d_in,
                             int64_t d_out, int64_t comps, int64_t groups, const int64_t* ptr, const int64_t* perm, int64_t ld_x,
                             int64_t ld_gout, int64_t ld_gx, int32_t dtype, void* workspace, size_t workspace_bytes, void* hip_stream) {
  cgtp::GroupedArgs a = {};
  a.x = x; a.W = W; a.gout = gout; a.gx = gx; a.gW = gW; a.gb = gb; a.ptr = ptr; a.perm = perm;
  a.rows = rows; a.d_in = d_in; a.d_out = d_out; a.comps = comps; a.groups = groups; a.ld_x = ld_x; a.ld_gout = ld_gout; a.ld_gx = ld_gx;
  cgtp_status s = check_grouped(a, dtype);
  if (s != CGTP_OK) return s;
  if (ld_x < comps * d_in || ld_gout < comps * d_out || ld_gx < comps * d_in) return fail(CGTP_EINVAL, "a row stride is smaller than its row");
  if (gb && comps != 1) return fail(CGTP_EINVAL, "biases are for rows of one component");
  if (groups == 0) return CGTP_OK;
  if (!gW || (rows > 0 && (!x || !W || !gout || !gx || !ptr))) return fail(CGTP_EINVAL, "NULL data pointer");
  s = check_numbers({x, W, gout, gx, gW, gb}, dtype);
  if (s != CGTP_OK) return s;
  if (!aligned(ptr, 8) || !aligned(perm, 8)) return fail(CGTP_EINVAL, "data pointers must be aligned to their type");
  hipStream_t st = (hipStream_t)hip_stream;
  if (rows == 0) {   // empty sums
    const size_t e = dtype == CGTP_F64 ? 8 : 4;
    HIP_TRY(cgtp::launch_fill_zero(gW, (size_t)(groups * d_in * d_out) * e, st));
    if (gb) HIP_TRY(cgtp::launch_fill_zero(gb, (size_t)(groups * d_out) * e, st));
    return CGTP_OK;
  }
  const size_t need = cgtp_grouped_workspace_bytes(rows, d_in, d_out, comps, groups, dtype);
  if (!workspace_serves(workspace, workspace_bytes, need)) return bad_workspace("cgtp_grouped_workspace_bytes", need);
  HIP_TRY((dtype == CGTP_F64 ? cgtp::grouped_backward_f64 : cgtp::grouped_backward_f32)(a, workspace, st));
  return CGTP_OK;
}

size_t cgtp_orthogonalise_workspace_bytes(int64_t batch, int64_t m, int64_t n, int32_t dtype) {
  if (check_orth(batch, m, n, dtype) != CGTP_OK || batch == 0) return 0;
  return (dtype == CGTP_F64 ? cgtp::orth_workspace_bytes_f64 : cgtp::orth_workspace_bytes_f32)(batch, m, n);
}

cgtp_status orthogonalise(const void* g, void* out, int64_t batch, int64_t m, int64_t n, int64_t ld_g, int64_t ld_out, int64_t stride_g,
                          int64_t stride_out, const double* coefficients, int32_t steps, double eps, int32_t dtype, void* workspace,
                          size_t workspace_bytes, void* hip_stream) {
  cgtp_status s = check_orth(batch, m, n, dtype);
  if (s != CGTP_OK) return s;
  if (ld_g < n || ld_out < n) return fail(CGTP_EINVAL, "a row stride is smaller than its row");
  if (stride_g < 0 || stride_out < 0) return fail(CGTP_EINVAL, "strides of matrices must not be negative");
  if (ld_g >= 1 << 22 || ld_out >= 1 << 22 || stride_g > ((int64_t)1 << 60) / std::max<int64_t>(batch, 1) ||
      stride_out > ((int64_t)1 << 60) / std::max<int64_t>(batch, 1))
    return fail(CGTP_EUNSUPPORTED, "row strides must be below 2^22, strides of matrices times batch below 2^60");
  // one behind the other, or side by side in wide rows
  if (batch > 1 && stride_out < (m - 1) * ld_out + n && (stride_out < n || ld_out < (batch - 1) * stride_out + n)) return fail(CGTP_EINVAL, "matrices of out overlap");
  if (steps < 1 || steps > 64) return fail(CGTP_EINVAL, "steps must be from 1 to 64");
  if (!coefficients) return fail(CGTP_EINVAL, "coefficients is NULL");
  for (int i = 0; i < 3 * steps; ++i)
    if (!std::isfinite(coefficients[i]) || (dtype == CGTP_F32 && std::fabs(coefficients[i]) > FLT_MAX)) return fail(CGTP_EINVAL, "coefficients must be finite numbers of the type");
  if (!(eps >= DBL_MIN && eps <= DBL_MAX)) return fail(CGTP_EINVAL, "eps must be a positive normal number");
  if (batch == 0) return CGTP_OK;
  if (!g || !out) return fail(CGTP_EINVAL, "NULL data pointer");
  s = check_numbers({g, out}, dtype);
  if (s != CGTP_OK) return s;
  const size_t need = cgtp_orthogonalise_workspace_bytes(batch, m, n, dtype);
  if (!workspace_serves(workspace, workspace_bytes, need)) return bad_workspace("cgtp_orthogonalise_workspace_bytes", need);
  cgtp::OrthArgs a = {g, out, batch, m, n, ld_g, ld_out, stride_g, stride_out, eps};
  HIP_TRY((dtype == CGTP_F64 ? cgtp::orth_f64 : cgtp::orth_f32)(a, coefficients, steps, workspace, (hipStream_t)hip_stream));
  return CGTP_OK;
}

}  // extern "C"
