// Dynamic LDS above 64 KiB has to be allowed for a kernel before its launch.
#pragma once

#include <hip/hip_runtime.h>

#include "lds_grant.h"

namespace bacon {

// Allows Kern `bytes` of dynamic LDS on the current device.
template <auto Kern>
static hipError_t allow_lds(size_t bytes) {
  static LdsGrants grants;
  if (bytes <= LdsGrants::kFree) return hipSuccess;
  int device = 0;
  const hipError_t e = hipGetDevice(&device);
  if (e != hipSuccess) return e;
  return (hipError_t)grants.grant(device, bytes, [](size_t b) {
    return (int)hipFuncSetAttribute(reinterpret_cast<const void *>(Kern), hipFuncAttributeMaxDynamicSharedMemorySize,
                                    (int)b);
  });
}

}  // namespace bacon
