// Host side shared by the calls that keep nothing (adapt.hip, heads.hip,
// spmm_grad.hip): errors, workspaces, and arrays that may not overlap.
#pragma once

#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstddef>
#include <cstdint>
#include <string>

#include "internal.h"

namespace spdp {

inline int hip_fail(hipError_t e, const char* what) {
  return fail(SPDP_ERR_HIP, std::string(what) + ": " + hipGetErrorString(e));
}

// the current device's
inline int compute_units(int* cus) {
  int dev = -1;
  hipError_t e = hipGetDevice(&dev);
  if (e != hipSuccess) return hip_fail(e, "hipGetDevice");
  e = hipDeviceGetAttribute(cus, hipDeviceAttributeMultiprocessorCount, dev);
  if (e != hipSuccess) return hip_fail(e, "hipDeviceGetAttribute");
  *cus = std::max(1, *cus);
  return SPDP_OK;
}

struct Array {
  const void* p;  // NULL: overlaps nothing
  size_t bytes;
};

inline bool overlap(const void* p, size_t np, const void* q, size_t nq) {
  const uintptr_t a = reinterpret_cast<uintptr_t>(p), b = reinterpret_cast<uintptr_t>(q);
  return p && q && a < b + nq && b < a + np;
}

// parts of a workspace start at multiples of 256 bytes
inline size_t aligned(size_t bytes) { return (bytes + 255) / 256 * 256; }

inline int check_workspace(const void* workspace, size_t have, size_t need) {
  if (need == 0) return SPDP_OK;
  if (!workspace) return fail(SPDP_ERR_INVALID_ARG, "workspace is NULL");
  if (reinterpret_cast<uintptr_t>(workspace) & 255) return fail(SPDP_ERR_INVALID_ARG, "workspace must be 256-byte aligned");
  if (have < need)
    return fail(SPDP_ERR_INVALID_ARG, "workspace of " + std::to_string(have) + " bytes, " + std::to_string(need) + " needed");
  return SPDP_OK;
}

// A call's body. No C++ exception leaves the ABI: a message may find no memory.
template <class F>
int guarded(F f) {
  try {
    clear_error();
    return f();
  } catch (...) {
    return SPDP_ERR_OOM;
  }
}

}  // namespace spdp
