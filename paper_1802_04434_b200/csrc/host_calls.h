// Host-side helpers of the calls around the step: arguments out of a block, shared memory of a kernel.
#ifndef SSGD_HOST_CALLS_H_
#define SSGD_HOST_CALLS_H_

#include "host_common.h"

namespace {

// A pointer out of a block of arguments.
template <typename T>
inline T* block_ptr(uint64_t word) { return reinterpret_cast<T*>(static_cast<uintptr_t>(word)); }

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

}  // namespace

#endif  // SSGD_HOST_CALLS_H_
