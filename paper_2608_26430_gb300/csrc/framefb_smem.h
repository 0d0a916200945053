// Dynamic shared memory limits of the library's kernels.  Internal: not part
// of the C ABI.
#pragma once
#include <cuda_runtime.h>
#include <stddef.h>

#include "framefb.h"

namespace ffb_host {

// Lets kernel `f` be launched with `smem` bytes of dynamic shared memory on
// the current device.  The limit belongs to the kernel, not to a call: a limit
// of one call's size may be lowered by another host thread before that call's
// launch, which then fails.  So a limit that is too low is raised to all that
// a block can have beside the kernel's static shared memory, and no limit is
// ever lowered (what a launch takes is its own argument).  The kernel is asked
// each time: the answer stays right after a device reset.
inline framefb_status allow_smem(const void* f, size_t smem) {
  cudaFuncAttributes at{};
  if (cudaFuncGetAttributes(&at, f) != cudaSuccess) return FRAMEFB_ECUDA;
  if (at.maxDynamicSharedSizeBytes >= 0 && static_cast<size_t>(at.maxDynamicSharedSizeBytes) >= smem) return FRAMEFB_OK;
  int dev = 0, most = 0;
  if (cudaGetDevice(&dev) != cudaSuccess ||
      cudaDeviceGetAttribute(&most, cudaDevAttrMaxSharedMemoryPerBlockOptin, dev) != cudaSuccess ||
      cudaFuncSetAttribute(f, cudaFuncAttributeMaxDynamicSharedMemorySize, most - static_cast<int>(at.sharedSizeBytes)) !=
          cudaSuccess)
    return FRAMEFB_ECUDA;
  return FRAMEFB_OK;
}

}  // namespace ffb_host
