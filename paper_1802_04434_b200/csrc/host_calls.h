// Host-side helpers of the calls around the step: arguments out of a block, shared memory of a kernel.
#ifndef SSGD_HOST_CALLS_H_
#define SSGD_HOST_CALLS_H_

#include <string.h>

#include "host_common.h"

namespace {

// A pointer out of a block of arguments.
template <typename T>
inline T* block_ptr(uint64_t word) { return reinterpret_cast<T*>(static_cast<uintptr_t>(word)); }

// A float out of a block: the bits of a double.
inline float block_float(uint64_t word) {
  double v;
  memcpy(&v, &word, sizeof v);
  return (float)v;
}

// Lets a kernel have `bytes` of dynamic shared memory, asked of the runtime once per kernel and device: `seen` is a
// static of the caller's, one for each kernel, a bit for each device.
inline bool allow_smem(const void* kernel, size_t bytes, unsigned long long* seen) {
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess) return false;
  const unsigned long long bit = dev >= 0 && dev < 64 ? 1ull << dev : 0;
  if (__atomic_load_n(seen, __ATOMIC_RELAXED) & bit) return true;
  if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)bytes) != cudaSuccess) return false;
  __atomic_fetch_or(seen, bit, __ATOMIC_RELAXED);
  return true;
}

// Whether a launch by clusters of more than eight CTAs has room on the current device, asked once per kernel and device.
inline bool allow_wide_clusters(const void* kernel, const cudaLaunchConfig_t& cfg, unsigned long long* seen) {
  int dev = 0, clusters = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 32) return false;
  const unsigned long long known = __atomic_load_n(seen, __ATOMIC_RELAXED) >> (2 * dev) & 3u;      // 2: asked, 1: there is room
  if (known & 2u) return known & 1u;
  const bool room = cudaFuncSetAttribute(kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1) == cudaSuccess &&
                    cudaOccupancyMaxActiveClusters(&clusters, kernel, &cfg) == cudaSuccess && clusters > 0;
  if (!room) (void)cudaGetLastError();
  __atomic_fetch_or(seen, (room ? 3ull : 2ull) << (2 * dev), __ATOMIC_RELAXED);
  return room;
}

}  // namespace

#endif  // SSGD_HOST_CALLS_H_
