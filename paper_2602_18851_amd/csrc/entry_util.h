// Host-side helpers of the entry points that need no context
// (spectral_quantize_fp8, spectral_matmul_fp8, spectral_rotary).
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>
#include <cstdio>

#include "spectral.h"

void sn_set_last_error(const char* msg);

namespace sn {

inline int refuse(int code, const char* msg) {
  sn_set_last_error(msg);
  return code;
}

// Whether the stream belongs to the current device (the default stream does).
inline int check_stream(hipStream_t st) {
  if (st == nullptr) return SN_OK;
  int cur = 0;
  hipDevice_t dev = 0;
  if (hipGetDevice(&cur) != hipSuccess || hipStreamGetDevice(st, &dev) != hipSuccess)
    return refuse(SN_EHIP, "the stream's device cannot be read");
  return dev == cur ? SN_OK : refuse(SN_ESTATE, "the stream does not belong to the current HIP device");
}

inline int launched(const char* what) {
  const hipError_t e = hipGetLastError();
  if (e == hipSuccess) return SN_OK;
  char buf[256];
  std::snprintf(buf, sizeof buf, "%s launch failed: %s", what, hipGetErrorString(e));
  return refuse(SN_EHIP, buf);
}

inline bool aligned(const void* p, uintptr_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }

}  // namespace sn
