// Tensor maps of asynchronous copies: the driver's encoder, found through the runtime so that the library needs no link to the driver.
#ifndef SSGD_TENSOR_MAP_H_
#define SSGD_TENSOR_MAP_H_

#include <cuda.h>
#include <cuda_runtime.h>

namespace {

typedef CUresult (*EncodeTiled)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*,
                                const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle,
                                CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
inline EncodeTiled encode_tiled() {
  static EncodeTiled cached = nullptr;          // any thread stores the same value
  EncodeTiled f = __atomic_load_n(&cached, __ATOMIC_RELAXED);
  if (f) return f;
  void* p = nullptr;
  cudaDriverEntryPointQueryResult found;
  if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &p, 12000, cudaEnableDefault, &found) != cudaSuccess ||
      found != cudaDriverEntryPointSuccess)
    return nullptr;
  f = reinterpret_cast<EncodeTiled>(p);
  __atomic_store_n(&cached, f, __ATOMIC_RELAXED);
  return f;
}

}  // namespace

#endif  // SSGD_TENSOR_MAP_H_
