// Entry points of the layer operators: the gated feed-forward block and the group normalisation.
#include <algorithm>
#include <atomic>
#include <cfloat>
#include <climits>
#include <memory>
#include <new>
#include <string>
#include <vector>

#include "csr.hpp"
#include "layer.hpp"
#include "norm.hpp"

struct cgtp_norm {
  cgtp::Norm N;
};

namespace {

using cgtp::fail;

#define HIP_TRY(expr)                                                                                   \
  do {                                                                                                  \
    hipError_t e_ = (expr);                                                                             \
    if (e_ != hipSuccess) return fail(CGTP_ERUNTIME, std::string(#expr) + ": " + hipGetErrorString(e_)); \
  } while (0)

bool aligned(const void* p, uintptr_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }

bool workspace_serves(const void* p, size_t have, size_t need) { return need == 0 || (p && have >= need && aligned(p, 256)); }

cgtp_status bad_workspace(const char* query, size_t need) {
  return fail(CGTP_EINVAL, "workspace: " + std::to_string(need) + " bytes needed (" + query + "), 256-byte aligned");
}

// compute units of the current device, asked for once
hipError_t compute_units(int& cus) {
  constexpr int kMaxDevices = 64;
  static std::atomic<int> known[kMaxDevices];
  int dev = -1;
  hipError_t e = hipGetDevice(&dev);
  if (e != hipSuccess) return e;
  if (dev < 0 || dev >= kMaxDevices) return hipErrorInvalidDevice;
  cus = known[dev].load(std::memory_order_relaxed);
  if (cus) return hipSuccess;
  e = hipDeviceGetAttribute(&cus, hipDeviceAttributeMultiprocessorCount, dev);
  cus = std::min(cus, 256);
  if (e == hipSuccess) known[dev].store(cus, std::memory_order_relaxed);
  return e;
}

cgtp_status check_gated(const cgtp::GatedArgs& a, int32_t dtype) {
  if (dtype != CGTP_F32 && dtype != CGTP_F64) return fail(CGTP_EINVAL, "dtype must be CGTP_F32 or CGTP_F64");
  if (a.act < CGTP_ACT_NONE || a.act > CGTP_ACT_TANH) return fail(CGTP_EINVAL, "unknown activation");
  if (a.rows < 0 || a.d_in <= 0 || a.d_out <= 0) return fail(CGTP_EINVAL, "rows must not be negative, d_in and d_out must be positive");
  if (a.rows > INT32_MAX) return fail(CGTP_EUNSUPPORTED, "rows must be below 2^31");
  if (a.d_in > 1 << 20 || a.d_out > 1 << 20 || a.d_in > INT32_MAX / a.d_out)
    return fail(CGTP_EUNSUPPORTED, "d_in and d_out must be at most 2^20, their product below 2^31");
  if ((a.bg == nullptr) != (a.bu == nullptr)) return fail(CGTP_EINVAL, "bg and bu must both be given or both be NULL");
  for (int64_t ld : {a.ld_x, a.ld_out, a.ld_gout, a.ld_gx})   // 64 rows are addressed with 31 bits
    if (ld >= 1 << 22) return fail(CGTP_EUNSUPPORTED, "row strides must be below 2^22");
  return CGTP_OK;
}

// How a call of the normalisation is cut up, and its workspace: the shares of long samples, partial sums of the parameters' gradients.
struct NormWork {
  int64_t R = 128, D = 0;   // rows of a short sample at most, of a chunk
  int64_t blocks = 1;       // workgroups (of each sub-unit)
  int64_t long_blocks = 1;  // of the second kernel
  int64_t sum_rows = 1;     // partial sums of the parameters' gradients (one: written where they belong at once)
  bool longer = false;      // samples of more than R rows are possible
  size_t part = 0, bytes = 0;
  NormWork(const cgtp::Norm& P, int64_t N, int64_t S, bool ptr, bool backward) {
    auto up = [](size_t v) { return (v + 255) / 256 * 256; };
    const size_t units = P.seg.size() * (size_t)P.groups;
    const int64_t most = 1 << 23;   // workgroups of a launch: 2^32 threads are too many (a normalisation has at most 2^14 sub-units)
    const bool any = P.call[(ptr ? cgtp::kGraphsForward : cgtp::kRowsForward) + backward].any;
    if (any) {
      // A workgroup has one unit of every so many samples.  Backward: as many workgroups as stay on the chip, each with a row of partial sums, but no more
      // than 256 MiB of them unless compute units would be without work (20 000 rows of 8192x0e fp32: 1630 us with 256 MiB, 2590 with 64)
      const int64_t groups = (int64_t)units, row = (P.n_w + P.n_b) * (int64_t)sizeof(double);
      const int64_t rows = backward ? std::max((256 + groups - 1) / groups, std::min(2048 / groups, ((int64_t)256 << 20) / row)) : (1 << 20) / groups;
      sum_rows = std::min(S, std::max<int64_t>(1, rows));
      blocks = sum_rows * groups;
    } else if (!ptr) {
      // Forward: a wave takes a step of rows; backward, where each workgroup leaves sums: as many workgroups as stay on the chip
      int rows = 1;
      for (const cgtp::NormSeg& s : P.seg) rows = std::max(rows, s.rows);
      const int64_t steps = (N + 4 * rows - 1) / (4 * rows);
      blocks = std::max<int64_t>(1, std::min<int64_t>(steps, std::max<int64_t>(1, (backward ? 2048 : most) / P.subs)));
      sum_rows = blocks;
    } else {
      // Chunks of 32 rows, of 64 where that leaves two workgroups a compute unit: a chunk's samples are found once (samples of 25 rows, l <= 3, 12 000 rows
      // of 32 channels forward and backward 67 us with 32 rows, 59 with 64, 58 with 128; l <= 2, 80 000 rows 165, 130 and 125; with 128 channels
      // 30 000 rows 407, 408 and 425); of 128 for long samples, whose shares each workgroup adds up
      D = N / 64 * P.subs >= 512 ? 64 : 32;
      if (N / 128 * P.subs >= 512 && N / 64 > 4 * S) {
        D = 128;
        // Longer ones where a sample has many: more workgroups than stay on the chip only add shares that each of them reads (one sample of 1 000 000 rows
        // of 128x0e in 32 groups, forward 1066 us with 128 rows, 489 with 512; 160 000 rows of 128 channels, l <= 3, 1014 and with 256 921; 16 samples in as
        // many rows 892 with 128, 927 with 256)
        while (N / D * P.subs > 2048 && N / D >= 256 * S) D *= 2;
      }
      while ((N + D - 1) / D > most / P.subs) D *= 2;
      R = std::max(R, D);
      const int64_t chunks = std::max<int64_t>(1, (N + D - 1) / D);
      longer = N > R;
      long_blocks = std::min<int64_t>(chunks, std::max(1, 2048 / P.subs));
      blocks = backward ? long_blocks : chunks;
      sum_rows = longer ? blocks + long_blocks : blocks;
      if (longer) part = up((size_t)chunks * 2 * units * 4 * sizeof(double));
    }
    bytes = part + (backward && (sum_rows > 1 || any) ? up((size_t)sum_rows * (size_t)(P.n_w + P.n_b) * sizeof(double)) : 0);
  }
};

// Compiles the kernels of the four calls, each with what fits it.  Registers that the code moves about are no place for a row's words (lanes of a
// wave are masked off in these kernels, and the compiler has been seen to move under a mask what all lanes need), and refused code is
// no code: such a call takes the kernels for any size.
void compile(cgtp::Norm& N) {
  bool any[2] = {};
  for (int i = 0; i < cgtp::kNormCalls; ++i) {
    cgtp::NormCall& c = N.call[i];
    try {
      cgtp::jit_compile(c.code, -2);
      c.any = c.any || c.code.relocates;
    } catch (const cgtp::RefusedCode&) {
      c.any = true;
    }
    if (c.any) c.code = cgtp::Kernel();
    any[i % 2] |= c.any;
  }
  for (int i = 0; i < 2; ++i) {
    if (!any[i]) N.any[i] = cgtp::Kernel();
    cgtp::jit_compile(N.any[i], -2);
    if (N.any[i].relocates) throw cgtp::RefusedCode(N.any[i].name + ": the compiled code relocates registers; the kernel is not used");
  }
}

hipFunction_t function(const cgtp::Kernel& k, const char* name) {
  hipFunction_t f = nullptr;
  const hipError_t e = hipModuleGetFunction(&f, k.module, name);
  if (e != hipSuccess) throw std::runtime_error(std::string("hipModuleGetFunction failed for ") + name + ": " + hipGetErrorString(e));
  return f;
}

void load(cgtp::Norm& N, int device) {
  for (int i = 0; i < cgtp::kNormCalls; ++i) {
    cgtp::NormCall& c = N.call[i];
    if (c.any) continue;
    cgtp::jit_compile(c.code, device);
    if (i == cgtp::kGraphsForward) c.longer = function(c.code, "cgtp_norm_long_fwd");
    if (i == cgtp::kGraphsBackward) c.longer = function(c.code, "cgtp_norm_long_bwd");
    if (i % 2) c.sums = function(c.code, "cgtp_norm_sums");
  }
  for (cgtp::Kernel& k : N.any) cgtp::jit_compile(k, device);
  if (N.any[1].module) N.any_sums = function(N.any[1], "cgtp_norm_sums");
  N.loaded = true;
}

void unload(cgtp::Norm& N) {
  for (cgtp::NormCall& c : N.call) cgtp::jit_unload(c.code);
  for (cgtp::Kernel& k : N.any) cgtp::jit_unload(k);
}

}  // namespace

extern "C" {

cgtp_status gated_forward(const void* x, const void* Wg, const void* Wu, const void* bg, const void* bu, void* out,
                          int64_t rows, int64_t d_in, int64_t d_out, int64_t ld_x, int64_t ld_out, int32_t act,
                          int32_t dtype, void* hip_stream) {
  cgtp::GatedArgs a = {};
  a.x = x; a.Wg = Wg; a.Wu = Wu; a.bg = bg; a.bu = bu; a.out = out;
  a.rows = rows; a.d_in = d_in; a.d_out = d_out; a.ld_x = ld_x; a.ld_out = ld_out; a.act = act;
  cgtp_status s = check_gated(a, dtype);
  if (s != CGTP_OK) return s;
  if (ld_x < d_in || ld_out < d_out) return fail(CGTP_EINVAL, "a row stride is smaller than its row");
  if (rows == 0) return CGTP_OK;
  if (!x || !Wg || !Wu || !out) return fail(CGTP_EINVAL, "NULL data pointer");
  for (const void* p : {x, Wg, Wu, bg, bu, (const void*)out})
    if (!aligned(p, 16)) return fail(CGTP_EINVAL, "data pointers must be 16-byte aligned");
  int cus = 0;
  HIP_TRY(compute_units(cus));
  HIP_TRY((dtype == CGTP_F64 ? cgtp::gated_forward_f64 : cgtp::gated_forward_f32)(a, cus, (hipStream_t)hip_stream));
  return CGTP_OK;
}

size_t cgtp_gated_workspace_bytes(int64_t rows, int64_t d_in, int64_t d_out, int32_t dtype) {
  cgtp::GatedArgs a = {};
  a.rows = rows; a.d_in = d_in; a.d_out = d_out;
  if (check_gated(a, dtype) != CGTP_OK || rows == 0) return 0;
  return (dtype == CGTP_F64 ? cgtp::gated_workspace_bytes_f64 : cgtp::gated_workspace_bytes_f32)(rows, d_in, d_out);
}

cgtp_status gated_backward(const void* x, const void* Wg, const void* Wu, const void* bg, const void* bu, const void* gout,
                           void* gx, void* gWg, void* gWu, void* gbg, void* gbu, int64_t rows, int64_t d_in, int64_t d_out,
                           int64_t ld_x, int64_t ld_gout, int64_t ld_gx, int32_t act, int32_t dtype, void* workspace,
                           size_t workspace_bytes, void* hip_stream) {
  cgtp::GatedArgs a = {};
  a.x = x; a.Wg = Wg; a.Wu = Wu; a.bg = bg; a.bu = bu; a.gout = gout; a.gx = gx; a.gWg = gWg; a.gWu = gWu; a.gbg = gbg; a.gbu = gbu;
  a.rows = rows; a.d_in = d_in; a.d_out = d_out; a.ld_x = ld_x; a.ld_gout = ld_gout; a.ld_gx = ld_gx; a.act = act;
  cgtp_status s = check_gated(a, dtype);
  if (s != CGTP_OK) return s;
  if (ld_x < d_in || ld_gout < d_out || ld_gx < d_in) return fail(CGTP_EINVAL, "a row stride is smaller than its row");
  if (!gWg || !gWu) return fail(CGTP_EINVAL, "NULL data pointer");
  if ((bg != nullptr) != (gbg != nullptr) || (bu != nullptr) != (gbu != nullptr))
    return fail(CGTP_EINVAL, "gbg and gbu must be given where bg and bu are, and be NULL where they are not");
  for (const void* p : {x, Wg, Wu, bg, bu, gout, (const void*)gx, (const void*)gWg, (const void*)gWu, (const void*)gbg, (const void*)gbu})
    if (!aligned(p, 16)) return fail(CGTP_EINVAL, "data pointers must be 16-byte aligned");
  hipStream_t st = (hipStream_t)hip_stream;
  if (rows == 0) {   // empty sums
    const size_t e = dtype == CGTP_F64 ? 8 : 4;
    HIP_TRY(cgtp::launch_fill_zero(gWg, (size_t)(d_in * d_out) * e, st));
    HIP_TRY(cgtp::launch_fill_zero(gWu, (size_t)(d_in * d_out) * e, st));
    if (gbg) {
      HIP_TRY(cgtp::launch_fill_zero(gbg, (size_t)d_out * e, st));
      HIP_TRY(cgtp::launch_fill_zero(gbu, (size_t)d_out * e, st));
    }
    return CGTP_OK;
  }
  if (!x || !Wg || !Wu || !gout || !gx) return fail(CGTP_EINVAL, "NULL data pointer");
  const size_t need = cgtp_gated_workspace_bytes(rows, d_in, d_out, dtype);
  if (!workspace_serves(workspace, workspace_bytes, need)) return bad_workspace("cgtp_gated_workspace_bytes", need);
  int cus = 0;
  HIP_TRY(compute_units(cus));
  HIP_TRY((dtype == CGTP_F64 ? cgtp::gated_backward_f64 : cgtp::gated_backward_f32)(a, cus, workspace, st));
  return CGTP_OK;
}

cgtp_status cgtp_norm_create(const char* irreps, int32_t groups, int32_t act, double eps, int32_t dtype, int32_t device,
                             uint32_t flags, cgtp_norm** out) {
  if (!out) return fail(CGTP_EINVAL, "out is NULL");
  *out = nullptr;
  if (!irreps) return fail(CGTP_EINVAL, "irreps string is NULL");
  if (flags & ~(uint32_t)(CGTP_IR_MUL | CGTP_NORM_GATED)) return fail(CGTP_EINVAL, "unknown bit in flags");
  if (dtype != CGTP_F32 && dtype != CGTP_F64) return fail(CGTP_EINVAL, "dtype must be CGTP_F32 or CGTP_F64");
  if (act < CGTP_ACT_NONE || act > CGTP_ACT_TANH) return fail(CGTP_EINVAL, "unknown activation");
  if (groups <= 0) return fail(CGTP_EINVAL, "the number of groups must be positive");
  const double least = dtype == CGTP_F64 ? DBL_MIN : FLT_MIN, greatest = dtype == CGTP_F64 ? DBL_MAX : FLT_MAX;
  if (!(eps >= least && eps <= greatest)) return fail(CGTP_EINVAL, "eps must be a positive normal number of the type");
  try {
    std::unique_ptr<cgtp_norm> H(new cgtp_norm());
    cgtp::Norm& N = H->N;
    std::vector<cgtp::Irrep> irs;
    try {
      irs = cgtp::parse_irreps(irreps);
    } catch (const std::invalid_argument& e) {
      return fail(CGTP_EINVAL, e.what());
    }
    if (irs.size() > 64) return fail(CGTP_EUNSUPPORTED, "more than 64 segments");
    N.groups = groups; N.act = act; N.eps = eps; N.dtype = dtype; N.device = device; N.ir_mul = flags & CGTP_IR_MUL;
    for (const cgtp::Irrep& ir : irs) {
      if (ir.l > cgtp::kMaxL) return fail(CGTP_EUNSUPPORTED, "l > 8");
      if (ir.mul > 65536) return fail(CGTP_EUNSUPPORTED, "multiplicity above 65536");
      if (ir.mul % groups != 0) return fail(CGTP_EINVAL, "the number of groups has to divide every multiplicity");
      cgtp::NormSeg s = {};
      s.mul = ir.mul;
      s.n = 2 * ir.l + 1;
      s.inv = ir.l == 0 && ir.p > 0;
      s.col = s.ycol = (int)N.dim_x;
      s.gate = s.gst = -1;
      s.st = (int)N.seg.size();
      s.w = (int)N.n_w;
      s.b = (int)N.n_b;
      N.dim_x += ir.dim();
      N.n_w += ir.mul;
      if (s.inv) N.n_b += ir.mul;
      N.seg.push_back(s);
    }
    N.dim_y = N.dim_x;
    int places = (int)N.seg.size();
    if (flags & CGTP_NORM_GATED)
      for (cgtp::NormSeg& s : N.seg)
        if (!s.inv) {
          s.gate = (int)N.dim_x;
          s.gst = places++;
          s.gw = (int)N.n_w;
          s.gb = (int)N.n_b;
          N.dim_x += s.mul;
          N.n_w += s.mul;
          N.n_b += s.mul;
        }
    N.n_stat = (int64_t)places * groups * 2;
    cgtp::emit_norm(N);
    // the kernels are loaded on `device`; the caller's current device is restored on return
    struct Restore {
      int device = -1;
      ~Restore() {
        if (device >= 0) (void)hipSetDevice(device);
      }
    } restore;
    if (device >= 0) {
      HIP_TRY(hipGetDevice(&restore.device));
      HIP_TRY(hipSetDevice(device));
      hipDeviceProp_t prop;
      HIP_TRY(hipGetDeviceProperties(&prop, device));
      N.num_cu = prop.multiProcessorCount;
      if (std::string(prop.gcnArchName).rfind("gfx950", 0) != 0)
        return fail(CGTP_EUNSUPPORTED, std::string("this library targets gfx950, device is ") + prop.gcnArchName);
    }
    try {
      if (device != -1) compile(N);
      if (device >= 0) load(N, device);
    } catch (const std::exception& e) {
      unload(N);
      return fail(CGTP_ECOMPILE, e.what());
    }
    *out = H.release();
    return CGTP_OK;
  } catch (const std::bad_alloc&) {
    return fail(CGTP_ENOMEM, "out of host memory");
  } catch (const std::exception& e) {
    return fail(CGTP_ERUNTIME, e.what());
  }
}

cgtp_status cgtp_norm_destroy(cgtp_norm* norm) {
  if (!norm) return CGTP_OK;
  unload(norm->N);
  delete norm;
  return CGTP_OK;
}

int64_t cgtp_norm_dim(const cgtp_norm* norm, int32_t which) {
  if (!norm) return -1;
  const cgtp::Norm& N = norm->N;
  switch (which) {
    case 0: return N.dim_x;
    case 1: return N.dim_y;
    case 2: return N.n_w;
    case 3: return N.n_b;
    case 4: return N.n_stat;
    default: return -1;
  }
}

const char* cgtp_norm_kernel(const cgtp_norm* norm, int32_t ptr, int32_t backward) {
  if (!norm) return nullptr;
  const int direction = backward != 0;
  const cgtp::NormCall& c = norm->N.call[(ptr ? cgtp::kGraphsForward : cgtp::kRowsForward) + direction];
  return (c.any ? norm->N.any[direction] : c.code).name.c_str();
}

size_t cgtp_norm_workspace_bytes(const cgtp_norm* norm, int64_t N, int64_t S, int32_t ptr, int32_t backward) {
  if (!norm || N < 0 || S < 0 || N > INT32_MAX || S > INT32_MAX || (!ptr && N != S) || S == 0) return 0;
  return NormWork(norm->N, N, S, ptr != 0, backward != 0).bytes;
}

}  // extern "C"

namespace {

cgtp_status check_norm(const cgtp_norm* norm, int64_t N, int64_t S, const int64_t* ptr, std::initializer_list<const void*> data) {
  if (!norm) return fail(CGTP_EINVAL, "norm is NULL");
  if (N < 0 || S < 0) return fail(CGTP_EINVAL, "negative size");
  if (!ptr && S != N) return fail(CGTP_EINVAL, "without ptr every row is a sample: S has to be N");
  if (N > INT32_MAX || S > INT32_MAX) return fail(CGTP_EUNSUPPORTED, "N and S must be below 2^31");
  for (const void* p : data)
    if (!aligned(p, 16)) return fail(CGTP_EINVAL, "data pointers must be 16-byte aligned");
  if (!norm->N.loaded) return fail(CGTP_EUNSUPPORTED, "the normalisation's kernels are not loaded (created without a device?)");
  int current = -1;      // its kernels are on one device
  HIP_TRY(hipGetDevice(&current));
  if (current != norm->N.device) return fail(CGTP_EINVAL, "the normalisation's device is not the current device");
  return CGTP_OK;
}

cgtp_status launch(hipFunction_t fn, int64_t grid, void** args, hipStream_t st, unsigned threads = 256) {
  HIP_TRY(hipModuleLaunchKernel(fn, (unsigned)grid, 1, 1, threads, 1, 1, 0, st, args, nullptr));
  return CGTP_OK;
}

}  // namespace

extern "C" {

cgtp_status norm_forward(const cgtp_norm* norm, const void* x, const void* weight, const void* bias, void* y, void* stats,
                         int64_t N, int64_t S, const int64_t* ptr, void* workspace, size_t workspace_bytes, void* hip_stream) {
  cgtp_status s = check_norm(norm, N, S, ptr, {x, weight, bias, y, stats});
  if (s != CGTP_OK) return s;
  if (S == 0) return CGTP_OK;
  const cgtp::Norm& P = norm->N;
  if ((N > 0 && (!x || !y)) || !weight || (P.n_b && !bias)) return fail(CGTP_EINVAL, "NULL data pointer");
  const NormWork w(P, N, S, ptr != nullptr, false);
  if (!workspace_serves(workspace, workspace_bytes, w.bytes)) return bad_workspace("cgtp_norm_workspace_bytes", w.bytes);
  hipStream_t st = (hipStream_t)hip_stream;
  double* part = (double*)workspace;
  const cgtp::NormCall& c = P.call[ptr ? cgtp::kGraphsForward : cgtp::kRowsForward];
  if (c.any) {
    void* args[] = {(void*)&x, (void*)&weight, (void*)&bias, (void*)&y, (void*)&stats, (void*)&N, (void*)&S, (void*)&ptr};
    return launch(P.any[0].fn, w.blocks, args, st);
  }
  if (!ptr) {
    void* args[] = {(void*)&x, (void*)&weight, (void*)&bias, (void*)&y, (void*)&stats, (void*)&N};
    return launch(c.code.fn, w.blocks * P.subs, args, st);
  }
  void* args[] = {(void*)&x, (void*)&weight, (void*)&bias, (void*)&y, (void*)&stats, (void*)&part, (void*)&ptr, (void*)&N, (void*)&S, (void*)&w.R, (void*)&w.D};
  s = launch(c.code.fn, w.blocks * P.subs, args, st);
  return s != CGTP_OK || !w.longer ? s : launch(c.longer, w.long_blocks * P.subs, args, st);
}

cgtp_status norm_backward(const cgtp_norm* norm, const void* x, const void* weight, const void* bias, const void* gy,
                          const void* stats, void* gx, void* gweight, void* gbias, int64_t N, int64_t S, const int64_t* ptr,
                          void* workspace, size_t workspace_bytes, void* hip_stream) {
  cgtp_status s = check_norm(norm, N, S, ptr, {x, weight, bias, gy, stats, gx, gweight, gbias});
  if (s != CGTP_OK) return s;
  const cgtp::Norm& P = norm->N;
  if (!gweight || (P.n_b && !gbias)) return fail(CGTP_EINVAL, "NULL data pointer");
  hipStream_t st = (hipStream_t)hip_stream;
  if (S == 0) {
    HIP_TRY(cgtp::launch_fill_zero(gweight, (size_t)P.n_w * P.elt(), st));
    if (P.n_b) HIP_TRY(cgtp::launch_fill_zero(gbias, (size_t)P.n_b * P.elt(), st));
    return CGTP_OK;
  }
  if ((N > 0 && (!x || !gy || !gx)) || !weight || (P.n_b && !bias) || !stats) return fail(CGTP_EINVAL, "NULL data pointer");
  const NormWork w(P, N, S, ptr != nullptr, true);
  if (!workspace_serves(workspace, workspace_bytes, w.bytes)) return bad_workspace("cgtp_norm_workspace_bytes", w.bytes);
  double* part = (double*)workspace;
  const cgtp::NormCall& c = P.call[ptr ? cgtp::kGraphsBackward : cgtp::kRowsBackward];
  double* sums = w.sum_rows > 1 || c.any ? (double*)((char*)workspace + w.part) : nullptr;
  if (c.any) {
    void* args[] = {(void*)&x, (void*)&weight, (void*)&bias, (void*)&gy, (void*)&stats, (void*)&gx, (void*)&sums, (void*)&N, (void*)&S, (void*)&ptr};
    s = launch(P.any[1].fn, w.blocks, args, st);
  } else if (!ptr) {
    void* args[] = {(void*)&x, (void*)&weight, (void*)&bias, (void*)&gy, (void*)&stats, (void*)&gx, (void*)&sums, (void*)&gweight, (void*)&gbias, (void*)&N};
    s = launch(c.code.fn, w.blocks * P.subs, args, st);
  } else {
    double* more = sums ? sums + w.blocks * (P.n_w + P.n_b) : nullptr;
    void* args[] = {(void*)&x, (void*)&weight, (void*)&bias, (void*)&gy, (void*)&stats, (void*)&gx, (void*)&part, (void*)&sums, (void*)&gweight, (void*)&gbias,
                    (void*)&ptr, (void*)&N, (void*)&S, (void*)&w.R, (void*)&w.D};
    s = launch(c.code.fn, w.blocks * P.subs, args, st);
    args[7] = (void*)&more;
    if (s == CGTP_OK && w.longer) s = launch(c.longer, w.long_blocks * P.subs, args, st);
  }
  if (s != CGTP_OK || !sums) return s;
  void* args[] = {(void*)&sums, (void*)&w.sum_rows, (void*)&gweight, (void*)&gbias};
  return launch(c.any ? P.any_sums : c.sums, (P.n_w + P.n_b + 15) / 16, args, st, 1024);
}

}  // extern "C"
