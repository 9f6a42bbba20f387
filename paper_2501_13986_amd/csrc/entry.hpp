// What the entry points of the layer operators and of the products share.
#pragma once

#include <hip/hip_runtime_api.h>

#include <algorithm>
#include <atomic>
#include <cstddef>
#include <cstdint>
#include <string>

#include "plan.hpp"

#define HIP_TRY(expr)                                                                                   \
  do {                                                                                                  \
    hipError_t e_ = (expr);                                                                             \
    if (e_ != hipSuccess) return cgtp::fail(CGTP_ERUNTIME, std::string(#expr) + ": " + hipGetErrorString(e_)); \
  } while (0)

namespace cgtp {

inline bool aligned(const void* p, uintptr_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }

inline bool workspace_serves(const void* p, size_t have, size_t need) { return need == 0 || (p && have >= need && aligned(p, 256)); }

inline cgtp_status bad_workspace(const char* query, size_t need) {
  return fail(CGTP_EINVAL, "workspace: " + std::to_string(need) + " bytes needed (" + query + "), 256-byte aligned");
}

// compute units of the current device, asked for once
inline hipError_t compute_units(int& cus) {
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

}  // namespace cgtp
