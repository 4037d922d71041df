// The element types of tensors around the step (fp32, bf16, fp16): sizes, conversions, accesses of four elements.
#ifndef SSGD_DTYPES_CUH_
#define SSGD_DTYPES_CUH_

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "signsgd.h"

namespace {

inline size_t dtype_bytes(unsigned type) {   // 0 for a type that the library does not know
  return type == SSGD_F32 ? 4 : type == SSGD_BF16 || type == SSGD_F16 ? 2 : 0;
}

__device__ __forceinline__ float to_float(float v) { return v; }
__device__ __forceinline__ float to_float(__nv_bfloat16 v) { return __bfloat162float(v); }
__device__ __forceinline__ float to_float(__half v) { return __half2float(v); }

template <typename T> __device__ __forceinline__ T from_float(float v);
template <> __device__ __forceinline__ float from_float<float>(float v) { return v; }
template <> __device__ __forceinline__ __nv_bfloat16 from_float<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }
template <> __device__ __forceinline__ __half from_float<__half>(float v) { return __float2half_rn(v); }

// Four consecutive elements; the address is a multiple of four elements.
__device__ __forceinline__ float4 load4(const float* p) { return *reinterpret_cast<const float4*>(p); }
__device__ __forceinline__ float4 load4(const __nv_bfloat16* p) {
  const uint2 v = *reinterpret_cast<const uint2*>(p);
  return make_float4(__uint_as_float(v.x << 16), __uint_as_float(v.x & 0xFFFF0000u), __uint_as_float(v.y << 16),
                     __uint_as_float(v.y & 0xFFFF0000u));
}
__device__ __forceinline__ float4 load4(const __half* p) {
  const uint2 v = *reinterpret_cast<const uint2*>(p);
  const float2 a = __half22float2(*reinterpret_cast<const __half2*>(&v.x));
  const float2 b = __half22float2(*reinterpret_cast<const __half2*>(&v.y));
  return make_float4(a.x, a.y, b.x, b.y);
}

// The two elements of a 32-bit word.
__device__ __forceinline__ float low_to_float(__nv_bfloat16, unsigned w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float high_to_float(__nv_bfloat16, unsigned w) { return __uint_as_float(w & 0xFFFF0000u); }
__device__ __forceinline__ float low_to_float(__half, unsigned w) { return __low2float(*reinterpret_cast<const __half2*>(&w)); }
__device__ __forceinline__ float high_to_float(__half, unsigned w) { return __high2float(*reinterpret_cast<const __half2*>(&w)); }
__device__ __forceinline__ float low_to_float(float, unsigned w) { return __uint_as_float(w); }
__device__ __forceinline__ float high_to_float(float, unsigned w) { return __uint_as_float(w); }

__device__ __forceinline__ unsigned pack2(__nv_bfloat16, float lo, float hi) {
  const __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
  return *reinterpret_cast<const unsigned*>(&v);
}
__device__ __forceinline__ unsigned pack2(__half, float lo, float hi) {
  const __half2 v = __floats2half2_rn(lo, hi);
  return *reinterpret_cast<const unsigned*>(&v);
}

__device__ __forceinline__ void store4(float* p, float4 v) { __stcs(reinterpret_cast<float4*>(p), v); }
template <typename T>
__device__ __forceinline__ void store4(T* p, float4 v) {
  __stcs(reinterpret_cast<uint2*>(p), make_uint2(pack2(T(), v.x, v.y), pack2(T(), v.z, v.w)));
}

// Eight consecutive elements; the address is a multiple of eight elements (for fp32 loads, of four).
__device__ __forceinline__ void load8(const float* p, float (&v)[8]) {
  const float4 a = *reinterpret_cast<const float4*>(p), b = *reinterpret_cast<const float4*>(p + 4);
  v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w; v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
}
template <typename T>
__device__ __forceinline__ void load8(const T* p, float (&v)[8]) {
  const uint4 q = *reinterpret_cast<const uint4*>(p);
  v[0] = low_to_float(T(), q.x); v[1] = high_to_float(T(), q.x); v[2] = low_to_float(T(), q.y); v[3] = high_to_float(T(), q.y);
  v[4] = low_to_float(T(), q.z); v[5] = high_to_float(T(), q.z); v[6] = low_to_float(T(), q.w); v[7] = high_to_float(T(), q.w);
}

}  // namespace

#endif  // SSGD_DTYPES_CUH_
