// Dynamic shared memory limits of the library's kernels.  Internal: not part
// of the C ABI.
#pragma once
#include <cuda_runtime.h>
#include <stdint.h>

#include <atomic>

#include "framefb.h"

namespace ffb_host {

// Lets kernel `f` be launched with all the dynamic shared memory that a block
// of the current device can have beside the kernel's static one.  The limit
// belongs to the kernel and the device, not to a call: a limit of one call's
// size may be lowered by another host thread before that call's launch, which
// then fails.  So it is raised to the most there is, once, and stays there
// (what a launch takes is its own argument).  Kernels that have been raised
// are kept in a table by address; one that finds no room in it is raised
// again with every call.
inline framefb_status allow_smem(const void* f) {
  constexpr int kDevices = 16, kBits = 9, kSlots = 1 << kBits;
  static std::atomic<const void*> raised[kDevices][kSlots];
  int dev = 0, most = 0;
  if (cudaGetDevice(&dev) != cudaSuccess) return FRAMEFB_ECUDA;
  const uint64_t h = (static_cast<uint64_t>(reinterpret_cast<uintptr_t>(f)) * 0x9E3779B97F4A7C15ull) >> (64 - kBits);
  std::atomic<const void*>* table = dev < kDevices ? raised[dev] : nullptr;
  if (table) {
    for (int i = 0; i < kSlots; ++i) {
      const void* p = table[(h + i) % kSlots].load(std::memory_order_acquire);
      if (p == f) return FRAMEFB_OK;
      if (!p) break;
    }
  }
  cudaFuncAttributes at{};
  if (cudaFuncGetAttributes(&at, f) != cudaSuccess ||
      cudaDeviceGetAttribute(&most, cudaDevAttrMaxSharedMemoryPerBlockOptin, dev) != cudaSuccess ||
      cudaFuncSetAttribute(f, cudaFuncAttributeMaxDynamicSharedMemorySize, most - static_cast<int>(at.sharedSizeBytes)) !=
          cudaSuccess)
    return FRAMEFB_ECUDA;
  if (table) {
    for (int i = 0; i < kSlots; ++i) {
      const void* p = nullptr;
      if (table[(h + i) % kSlots].compare_exchange_strong(p, f, std::memory_order_acq_rel) || p == f) break;
    }
  }
  return FRAMEFB_OK;
}

}  // namespace ffb_host
