// Quantisation to microscaled 4-bit numbers, by rows and by columns, and its inverse.  See include/signsgd.h.
//
//   mx: S = 2^(floor(log2 max|x|) - 2) over a block;   nv: S = max(e4m3(max|x| / t / 6), 2^-9) * t, t the tensor scale
//   code = nearest 4-bit value to x / S, ties to the even code, magnitudes above 6 to 6
// A block that holds an infinity or a NaN gets the NaN scale: it reads back as NaN, and so do products with it.

#include "host_common.h"
#include "dtypes.cuh"
#include "fp4.cuh"

namespace {

__device__ __forceinline__ unsigned magnitude_bits(float v) { return __float_as_uint(v) & 0x7FFFFFFFu; }

// Largest magnitude of a matrix, as ordered bits (NaN above infinity); `out` starts at 0.
template <typename T>
__global__ void __launch_bounds__(kThreads)
fp4_amax_kernel(const T* __restrict__ x, unsigned rows, unsigned cols, size_t ldx, unsigned* __restrict__ out) {
  unsigned top = 0;
  for (unsigned r = blockIdx.y; r < rows; r += gridDim.y) {
    const T* row = x + (size_t)r * ldx;
    for (unsigned c = blockIdx.x * kThreads + threadIdx.x; c < cols; c += gridDim.x * kThreads)
      top = max(top, magnitude_bits(to_float(row[c])));
  }
  top = __reduce_max_sync(0xFFFFFFFFu, top);
  if ((threadIdx.x & 31u) == 0) atomicMax(out, top);   // a maximum does not depend on the order
}

// x / s rounded to nearest, from the correctly rounded reciprocal r of s: one Newton correction of the product
// (Markstein, "Computation of elementary functions on the IBM RISC System/6000", 1990).  In this order of signs a
// quotient of -0 stays -0.
__device__ __forceinline__ float quotient(float x, float s, float r) {
  const float q = __fmul_rn(x, r);
  return __fmaf_rn(__fmaf_rn(q, s, -x), -r, q);
}

// Eight values to the four bytes of their codes: nearest, ties to even, saturating.
__device__ __forceinline__ unsigned fp4_pack8(const float* v) {
  unsigned out;
  asm("{\n\t.reg .b8 b0, b1, b2, b3;\n\t"
      "cvt.rn.satfinite.e2m1x2.f32 b0, %2, %1;\n\t"
      "cvt.rn.satfinite.e2m1x2.f32 b1, %4, %3;\n\t"
      "cvt.rn.satfinite.e2m1x2.f32 b2, %6, %5;\n\t"
      "cvt.rn.satfinite.e2m1x2.f32 b3, %8, %7;\n\t"
      "mov.b32 %0, {b0, b1, b2, b3};\n\t}"
      : "=r"(out)
      : "f"(v[0]), "f"(v[1]), "f"(v[2]), "f"(v[3]), "f"(v[4]), "f"(v[5]), "f"(v[6]), "f"(v[7]));
  return out;
}

// Scale byte of a block, and the two factors that bring its values to 4-bit range: x * pre / scale.
struct BlockScale {
  unsigned byte;
  float pre;      // power of two
  float scale;    // what is left to divide by (1 for mx)
  float inverse;  // its reciprocal
};
template <int FORMAT>
__device__ __forceinline__ BlockScale block_scale(unsigned top_bits, float tensor_scale) {
  BlockScale b;
  b.scale = b.inverse = 1.0f;
  if constexpr (FORMAT == SSGD_MXFP4) {
    // exponent of max|x| minus 2, kept at -127 or above (a block of zeros or subnormals)
    const int e = (int)(top_bits >> 23) - 2;
    b.byte = top_bits >= 0x7F800000u ? 255u : (unsigned)max(e, 0);
    b.pre = b.byte >= 254u ? __uint_as_float(0x00400000u) : __uint_as_float((254u - b.byte) << 23);   // 2^(127 - byte)
  } else {
    b.pre = __fdiv_rn(1.0f, tensor_scale);
    const float s = __fdiv_rn(__fmul_rn(__uint_as_float(top_bits), b.pre), 6.0f);
    const __nv_fp8_storage_t q = __nv_cvt_float_to_fp8(fminf(s, 448.0f), __NV_SATFINITE, __NV_E4M3);
    b.byte = top_bits >= 0x7F800000u ? 0x7Fu : max((unsigned)q, 1u);   // 1 = 2^-9, the least positive
    if (b.byte != 0x7Fu) b.scale = e4m3_value(b.byte);
    b.inverse = __frcp_rn(b.scale);
  }
  return b;
}
template <int FORMAT>
__device__ __forceinline__ float scaled(float v, const BlockScale& b) {
  v = __fmul_rn(v, b.pre);
  return FORMAT == SSGD_MXFP4 ? v : quotient(v, b.scale, b.inverse);
}

// One thread, one block: `vec` consecutive values along the block, at a stride of `step` elements.
template <int FORMAT, typename T>
__device__ __forceinline__ void quantise_block(const T* __restrict__ x, size_t step, unsigned n, float tensor_scale,
                                               uint8_t* __restrict__ codes, uint8_t* __restrict__ scale_byte) {
  constexpr int B = FORMAT == SSGD_MXFP4 ? 32 : 16;
  float v[B];
  unsigned top = 0;
#pragma unroll
  for (int i = 0; i < B; ++i) {
    v[i] = (unsigned)i < n ? to_float(x[i * step]) : 0.0f;
    top = max(top, magnitude_bits(v[i]));
  }
  const BlockScale b = block_scale<FORMAT>(top, tensor_scale);
  const bool finite = top < 0x7F800000u;
  if (FORMAT == SSGD_NVFP4 && finite && __uint_as_float(top) * b.pre > 1e30f) {   // a tensor scale far too small: saturate
#pragma unroll
    for (int i = 0; i < B; ++i) v[i] = fmaxf(-1e30f / b.pre, fminf(1e30f / b.pre, v[i]));
  }
#pragma unroll
  for (int i = 0; i < B; ++i) v[i] = scaled<FORMAT>(v[i], b);
#pragma unroll
  for (int w = 0; w < B / 8; ++w) reinterpret_cast<uint32_t*>(codes)[w] = finite ? fp4_pack8(v + 8 * w) : 0u;
  *scale_byte = n ? (uint8_t)b.byte : 0;
}

// TRANSPOSED: rows of the result are columns of x.  Lanes run along x's columns in both cases.
template <int FORMAT, bool TRANSPOSED, typename T>
__global__ void __launch_bounds__(kThreads)
fp4_quantise_kernel(const T* __restrict__ x, unsigned rows, unsigned cols, size_t ldx, const float* __restrict__ amax,
                    float* __restrict__ tensor_scale, uint8_t* __restrict__ codes, uint8_t* __restrict__ scales) {
  constexpr unsigned B = FORMAT == SSGD_MXFP4 ? 32 : 16;
  const float ts = FORMAT == SSGD_NVFP4 ? fp4_tensor_scale(__ldg(amax)) : 1.0f;
  if (FORMAT == SSGD_NVFP4 && blockIdx.x == 0 && threadIdx.x == 0) tensor_scale[0] = ts;
  const unsigned out_rows = TRANSPOSED ? cols : rows, out_cols = TRANSPOSED ? rows : cols;
  const size_t row_bytes = (size_t)((out_cols + 31) / 32) * 16;
  const size_t tiles_k = ((out_cols + B - 1) / B + 3) / 4;
  const size_t padded_blocks = tiles_k * 4, padded_rows = (size_t)(out_rows + 127) / 128 * 128;
  const size_t total = padded_blocks * padded_rows;
  for (size_t i = (size_t)blockIdx.x * kThreads + threadIdx.x; i < total; i += (size_t)gridDim.x * kThreads) {
    const unsigned row = (unsigned)(TRANSPOSED ? i % padded_rows : i / padded_blocks);
    const unsigned block = (unsigned)(TRANSPOSED ? i / padded_rows : i % padded_blocks);
    uint8_t* sb = scales + fp4_scale_index(row, block, tiles_k);
    const unsigned c0 = block * B;
    if (row >= out_rows || (size_t)c0 >= row_bytes * 2) {   // padding of the scale tiles
      *sb = 0;
      continue;
    }
    const unsigned n = c0 >= out_cols ? 0u : min(B, out_cols - c0);
    const T* src = TRANSPOSED ? x + (size_t)c0 * ldx + row : x + (size_t)row * ldx + c0;
    quantise_block<FORMAT>(n ? src : x, TRANSPOSED ? ldx : 1, n, ts, codes + (size_t)row * row_bytes + c0 / 2, sb);
  }
}

template <int FORMAT, typename T>
__global__ void __launch_bounds__(kThreads)
fp4_dequantise_kernel(const uint8_t* __restrict__ codes, const uint8_t* __restrict__ scales, const float* __restrict__ tensor_scale,
                      unsigned rows, unsigned cols, T* __restrict__ out, size_t ldo) {
  constexpr unsigned B = FORMAT == SSGD_MXFP4 ? 32 : 16;
  const float ts = FORMAT == SSGD_NVFP4 && tensor_scale ? __ldg(tensor_scale) : 1.0f;
  const size_t row_bytes = (size_t)((cols + 31) / 32) * 16;
  const unsigned quads = (cols + 3) / 4;
  const size_t tiles_k = ((cols + B - 1) / B + 3) / 4, total = (size_t)rows * quads;
  for (size_t i = (size_t)blockIdx.x * kThreads + threadIdx.x; i < total; i += (size_t)gridDim.x * kThreads) {
    const unsigned row = (unsigned)(i / quads), c = (unsigned)(i % quads) * 4;
    const unsigned four = *reinterpret_cast<const uint16_t*>(codes + (size_t)row * row_bytes + c / 2);
    const float s = __fmul_rn(fp4_scale_value<FORMAT>(scales[fp4_scale_index(row, c / B, tiles_k)]), ts);
#pragma unroll
    for (unsigned j = 0; j < 4; ++j)
      if (c + j < cols) out[(size_t)row * ldo + c + j] = from_float<T>(__fmul_rn(fp4_value(four >> (4 * j)), s));
  }
}

unsigned grid_of(size_t threads) {
  const size_t ctas = (threads + kThreads - 1) / kThreads;
  return (unsigned)(ctas < 1 ? 1 : ctas < (1u << 20) ? ctas : (1u << 20));
}

template <int FORMAT, typename T>
void launch_quantise(const T* x, size_t rows, size_t cols, size_t ldx, const float* amax, float* tensor_scale, uint8_t* codes,
                     uint8_t* scales, uint8_t* codes_t, uint8_t* scales_t, cudaStream_t s) {
  const unsigned r = (unsigned)rows, c = (unsigned)cols;
  if (codes)
    fp4_quantise_kernel<FORMAT, false><<<grid_of(ssgd_fp4_scale_bytes(FORMAT, rows, cols)), kThreads, 0, s>>>(x, r, c, ldx, amax, tensor_scale, codes, scales);
  if (codes_t)
    fp4_quantise_kernel<FORMAT, true><<<grid_of(ssgd_fp4_scale_bytes(FORMAT, cols, rows)), kThreads, 0, s>>>(x, r, c, ldx, amax, tensor_scale, codes_t, scales_t);
}

template <typename T>
ssgd_status quantise_typed(const T* x, size_t rows, size_t cols, size_t ldx, int format, const float* amax, float* tensor_scale,
                           uint8_t* codes, uint8_t* scales, uint8_t* codes_t, uint8_t* scales_t, cudaStream_t s) {
  if (format == SSGD_NVFP4 && !amax) {
    if (cudaMemsetAsync(tensor_scale + 1, 0, sizeof(float), s) != cudaSuccess) return SSGD_ERR_CUDA;
    const dim3 grid((unsigned)((cols + kThreads - 1) / kThreads < 64 ? (cols + kThreads - 1) / kThreads : 64), (unsigned)(rows < 1024 ? rows : 1024));
    fp4_amax_kernel<<<grid, kThreads, 0, s>>>(x, (unsigned)rows, (unsigned)cols, ldx, reinterpret_cast<unsigned*>(tensor_scale + 1));
    amax = tensor_scale + 1;
  }
  if (format == SSGD_MXFP4)
    launch_quantise<SSGD_MXFP4>(x, rows, cols, ldx, amax, tensor_scale, codes, scales, codes_t, scales_t, s);
  else
    launch_quantise<SSGD_NVFP4>(x, rows, cols, ldx, amax, tensor_scale, codes, scales, codes_t, scales_t, s);
  return launch_status();
}

template <int FORMAT>
void launch_dequantise(const uint8_t* codes, const uint8_t* scales, const float* ts, size_t rows, size_t cols, void* out, int dtype,
                       size_t ldo, cudaStream_t s) {
  const unsigned r = (unsigned)rows, c = (unsigned)cols, grid = grid_of(rows * ((cols + 3) / 4));
  switch (dtype) {
    case SSGD_F32: fp4_dequantise_kernel<FORMAT><<<grid, kThreads, 0, s>>>(codes, scales, ts, r, c, static_cast<float*>(out), ldo); break;
    case SSGD_BF16: fp4_dequantise_kernel<FORMAT><<<grid, kThreads, 0, s>>>(codes, scales, ts, r, c, static_cast<__nv_bfloat16*>(out), ldo); break;
    default: fp4_dequantise_kernel<FORMAT><<<grid, kThreads, 0, s>>>(codes, scales, ts, r, c, static_cast<__half*>(out), ldo); break;
  }
}

}  // namespace

extern "C" {

size_t ssgd_fp4_row_bytes(size_t cols) { return cols / 32 * 16 + (cols % 32 ? 16 : 0); }

size_t ssgd_fp4_scale_bytes(int format, size_t rows, size_t cols) {
  if (!fp4_format_ok(format) || rows > SSGD_FP4_MAX_SIDE || cols > SSGD_FP4_MAX_SIDE) return 0;
  return (rows + 127) / 128 * ((fp4_block_count(format, cols) + 3) / 4) * 512;
}

ssgd_status ssgd_fp4_quantise(const void* x, int dtype, size_t rows, size_t cols, size_t ldx, int format, const float* amax,
                              float* tensor_scale, uint8_t* codes, uint8_t* scales, uint8_t* codes_t, uint8_t* scales_t, void* stream) {
  if (!fp4_format_ok(format) || dtype_bytes((unsigned)dtype) == 0) return SSGD_ERR_ARG;
  if (!x || (!codes && !codes_t) || (codes && !scales) || (codes_t && !scales_t)) return SSGD_ERR_NULL;
  if (format == SSGD_NVFP4 && !tensor_scale) return SSGD_ERR_NULL;
  if (rows > SSGD_FP4_MAX_SIDE || cols > SSGD_FP4_MAX_SIDE || ldx < cols || mul_overflows(rows, ldx) || mul_overflows(rows * ldx, 4)) return SSGD_ERR_SIZE;
  if (reinterpret_cast<uintptr_t>(x) % dtype_bytes((unsigned)dtype) != 0 || !aligned16(codes) || !aligned16(scales) || !aligned16(codes_t) ||
      !aligned16(scales_t) || ((reinterpret_cast<uintptr_t>(amax) | reinterpret_cast<uintptr_t>(tensor_scale)) & 3u))
    return SSGD_ERR_ALIGN;
  if (rows == 0 || cols == 0) return SSGD_OK;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  switch (dtype) {
    case SSGD_F32: return quantise_typed(static_cast<const float*>(x), rows, cols, ldx, format, amax, tensor_scale, codes, scales, codes_t, scales_t, s);
    case SSGD_BF16: return quantise_typed(static_cast<const __nv_bfloat16*>(x), rows, cols, ldx, format, amax, tensor_scale, codes, scales, codes_t, scales_t, s);
    default: return quantise_typed(static_cast<const __half*>(x), rows, cols, ldx, format, amax, tensor_scale, codes, scales, codes_t, scales_t, s);
  }
}

ssgd_status ssgd_fp4_dequantise(const uint8_t* codes, const uint8_t* scales, const float* tensor_scale, int format, size_t rows,
                                size_t cols, void* out, int dtype, size_t ldo, void* stream) {
  if (!fp4_format_ok(format) || dtype_bytes((unsigned)dtype) == 0) return SSGD_ERR_ARG;
  if (!codes || !scales || !out) return SSGD_ERR_NULL;
  if (rows > SSGD_FP4_MAX_SIDE || cols > SSGD_FP4_MAX_SIDE || ldo < cols || mul_overflows(rows, ldo) || mul_overflows(rows * ldo, 4)) return SSGD_ERR_SIZE;
  if (!aligned16(codes) || !aligned16(scales) || reinterpret_cast<uintptr_t>(out) % dtype_bytes((unsigned)dtype) != 0 ||
      (reinterpret_cast<uintptr_t>(tensor_scale) & 3u))
    return SSGD_ERR_ALIGN;
  if (rows == 0 || cols == 0) return SSGD_OK;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  if (format == SSGD_MXFP4) launch_dequantise<SSGD_MXFP4>(codes, scales, tensor_scale, rows, cols, out, dtype, ldo, s);
  else launch_dequantise<SSGD_NVFP4>(codes, scales, tensor_scale, rows, cols, out, dtype, ldo, s);
  return launch_status();
}

}  // extern "C"
