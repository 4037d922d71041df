// Microscaled 4-bit numbers: what quantisation, its inverse and the product share.
//
// A value is sign, two exponent bits, one fraction bit: 0, 0.5, 1, 1.5, 2, 3, 4, 6.  A block of a row shares a scale:
//   SSGD_MXFP4  32 values and a power of two (one byte, exponent + 127; 255 = NaN)
//   SSGD_NVFP4  16 values and an E4M3 number (one byte; 0x7F = NaN); a tensor scale, a power of two, multiplies all
// Codes lie two in a byte, the even column in the low half, a row padded with zero codes to a multiple of 32 columns (16
// bytes).  Scale bytes lie in tiles of 128 rows x 4 blocks, the order in which the tensor cores take them: byte
// (row % 32) * 16 + (row / 32) * 4 + block % 4 of a tile's 512, tiles of the same rows one after another.
#ifndef SSGD_FP4_CUH_
#define SSGD_FP4_CUH_

#include <cuda_fp16.h>
#include <cuda_fp8.h>
#include <stdint.h>

#include "signsgd.h"

namespace {

constexpr int kFp4Block[2] = {32, 16};     // values of a block by format

inline bool fp4_format_ok(int format) { return format == SSGD_MXFP4 || format == SSGD_NVFP4; }
inline size_t fp4_block_count(int format, size_t cols) { return (cols + kFp4Block[format] - 1) / kFp4Block[format]; }

// Byte of the scale of (row, block); tiles_k = tiles of one row of tiles.
__host__ __device__ __forceinline__ size_t fp4_scale_index(size_t row, size_t block, size_t tiles_k) {
  return ((row >> 7) * tiles_k + (block >> 2)) * 512 + (row & 31) * 16 + ((row >> 5) & 3) * 4 + (block & 3);
}

// The two values of a byte of codes, the low half's first.
__device__ __forceinline__ float2 fp4_pair_value(unsigned byte) {
  unsigned h;
  asm("{\n\t.reg .b8 b0, b1, b2, b3;\n\tmov.b32 {b0, b1, b2, b3}, %1;\n\tcvt.rn.f16x2.e2m1x2 %0, b0;\n\t}" : "=r"(h) : "r"(byte));
  return __half22float2(*reinterpret_cast<const __half2*>(&h));
}

__device__ __forceinline__ float e8m0_value(unsigned byte) {
  if (byte == 255u) return __uint_as_float(0x7FC00000u);
  return __uint_as_float(byte == 0 ? 0x00400000u : byte << 23);
}
__device__ __forceinline__ float e4m3_value(unsigned byte) {
  const __half_raw h = __nv_cvt_fp8_to_halfraw((__nv_fp8_storage_t)byte, __NV_E4M3);
  return __half2float(__half(h));
}

// The scale of one block from its byte, without the tensor scale.
template <int FORMAT>
__device__ __forceinline__ float fp4_scale_value(unsigned byte) {
  return FORMAT == SSGD_MXFP4 ? e8m0_value(byte) : e4m3_value(byte);
}

// Least power of two t with 2688 t >= top (2688 = 6 * 448, the largest value times the largest scale): with
// top = m 2^e, 1 <= m < 2, and 2688 = 1.3125 * 2^11 that is 2^(e - 11), or 2^(e - 10) for m > 1.3125.  Exponent
// clamped to -100 .. 120; 1 for a top of zero, infinity or NaN.
__device__ __forceinline__ float fp4_tensor_scale(float top) {
  const unsigned u = __float_as_uint(top);
  if (!(top > 0.0f) || u >= 0x7F800000u) return 1.0f;
  int e = u < 0x00800000u ? -126 : (int)(u >> 23) - 127 - ((u & 0x7FFFFFu) > 0x280000u ? 10 : 11);
  e = max(-100, min(120, e));
  return __uint_as_float((unsigned)(e + 127) << 23);
}

}  // namespace

#endif  // SSGD_FP4_CUH_
