// Errors and device selection, shared by the entry points' files.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>
#include <string>

#include "csg.h"

namespace csg {

extern thread_local std::string g_last_error;  // what csg_last_error returns

// Sets the thread's message and returns s.
csg_status fail(csg_status s, const char* fmt, ...);

inline csg_status hip_fail(hipError_t e, const char* what) {
  return fail(e == hipErrorOutOfMemory ? CSG_ERR_NOMEM : CSG_ERR_HIP, "%s: %s", what, hipGetErrorString(e));
}

#define CSG_HIP(expr)                                       \
  do {                                                      \
    hipError_t e_ = (expr);                                 \
    if (e_ != hipSuccess) return csg::hip_fail(e_, #expr);  \
  } while (0)

// Restores the caller's current device on scope exit.
struct DeviceGuard {
  int prev = -1;
  hipError_t err = hipSuccess;
  explicit DeviceGuard(int dev) {
    err = hipGetDevice(&prev);
    if (err == hipSuccess && prev != dev) err = hipSetDevice(dev);
  }
  ~DeviceGuard() {
    if (prev >= 0) (void)hipSetDevice(prev);
  }
};

// Compute units of `device`, checked once to be the one this library is built for.
csg_status device_cus(int device, int32_t* cus);

inline bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

}  // namespace csg
