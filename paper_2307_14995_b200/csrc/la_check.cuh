// Checks that the entry points share.
#pragma once
#include <cuda_runtime.h>
#include <stdint.h>

#include "../../include/la.h"

namespace la {

inline bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

inline la_status check_device() {
  int dev = 0, major = 0;
  if (cudaGetDevice(&dev) != cudaSuccess) return LA_ERR_CUDA;
  if (cudaDeviceGetAttribute(&major, cudaDevAttrComputeCapabilityMajor, dev) != cudaSuccess)
    return LA_ERR_CUDA;
  return major == 10 ? LA_OK : LA_ERR_ARCH;
}

#define LA_TRY_CUDA(expr)                       \
  do {                                          \
    if ((expr) != cudaSuccess) return LA_ERR_CUDA; \
  } while (0)

}  // namespace la
