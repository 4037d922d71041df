// Product of two microscaled 4-bit operands, out[i][j] = sum_k A[i][k] B[j][k].  See include/signsgd.h.

#include "host_common.h"
#include "dtypes.cuh"
#include "fp4.cuh"

namespace {

// One output per thread, a 16 x 16 tile per CTA, 32 columns of k at a time through shared memory.
template <int FORMAT, typename T>
__global__ void __launch_bounds__(kThreads)
fp4_matmul_kernel(const uint8_t* __restrict__ a, const uint8_t* __restrict__ a_scales, const float* __restrict__ a_ts,
                  const uint8_t* __restrict__ b, const uint8_t* __restrict__ b_scales, const float* __restrict__ b_ts,
                  unsigned M, unsigned N, unsigned K, T* __restrict__ out, size_t ldo) {
  constexpr unsigned B = FORMAT == SSGD_MXFP4 ? 32 : 16;
  __shared__ float va[16][33], vb[16][33];
  const size_t row_bytes = (size_t)((K + 31) / 32) * 16, tiles_k = ((K + B - 1) / B + 3) / 4;
  const unsigned tx = threadIdx.x & 15u, ty = threadIdx.x >> 4;
  const unsigned tiles_n = (N + 15) / 16;
  const unsigned i0 = (unsigned)(blockIdx.x / tiles_n) * 16, j0 = (unsigned)(blockIdx.x % tiles_n) * 16;
  float acc = 0.0f;
  for (unsigned k0 = 0; k0 < row_bytes * 2; k0 += 32) {
    const unsigned k = k0 + tx * 2;
    const unsigned ra = i0 + ty, rb = j0 + ty;
    const unsigned ca = ra < M ? a[(size_t)ra * row_bytes + k / 2] : 0u, cb = rb < N ? b[(size_t)rb * row_bytes + k / 2] : 0u;
    const float sa = ra < M ? fp4_scale_value<FORMAT>(a_scales[fp4_scale_index(ra, k / B, tiles_k)]) : 0.0f;
    const float sb = rb < N ? fp4_scale_value<FORMAT>(b_scales[fp4_scale_index(rb, k / B, tiles_k)]) : 0.0f;
    va[ty][tx * 2] = fp4_value(ca & 15u) * sa; va[ty][tx * 2 + 1] = fp4_value(ca >> 4) * sa;
    vb[ty][tx * 2] = fp4_value(cb & 15u) * sb; vb[ty][tx * 2 + 1] = fp4_value(cb >> 4) * sb;
    __syncthreads();
#pragma unroll
    for (int q = 0; q < 32; ++q) acc = __fmaf_rn(va[ty][q], vb[tx][q], acc);
    __syncthreads();
  }
  const float ts = (a_ts ? __ldg(a_ts) : 1.0f) * (b_ts ? __ldg(b_ts) : 1.0f);
  if (i0 + ty < M && j0 + tx < N) out[(size_t)(i0 + ty) * ldo + j0 + tx] = from_float<T>(acc * ts);
}

template <int FORMAT>
void launch_matmul(const uint8_t* a, const uint8_t* as, const float* ats, const uint8_t* b, const uint8_t* bs, const float* bts, size_t M,
                   size_t N, size_t K, void* out, int dtype, size_t ldo, cudaStream_t s) {
  const unsigned m = (unsigned)M, n = (unsigned)N, k = (unsigned)K, grid = (unsigned)(((M + 15) / 16) * ((N + 15) / 16));
  switch (dtype) {
    case SSGD_F32: fp4_matmul_kernel<FORMAT><<<grid, kThreads, 0, s>>>(a, as, ats, b, bs, bts, m, n, k, static_cast<float*>(out), ldo); break;
    case SSGD_BF16: fp4_matmul_kernel<FORMAT><<<grid, kThreads, 0, s>>>(a, as, ats, b, bs, bts, m, n, k, static_cast<__nv_bfloat16*>(out), ldo); break;
    default: fp4_matmul_kernel<FORMAT><<<grid, kThreads, 0, s>>>(a, as, ats, b, bs, bts, m, n, k, static_cast<__half*>(out), ldo); break;
  }
}

}  // namespace

extern "C" {

ssgd_status ssgd_fp4_matmul(const uint8_t* a_codes, const uint8_t* a_scales, const float* a_tensor_scale, const uint8_t* b_codes,
                            const uint8_t* b_scales, const float* b_tensor_scale, size_t M, size_t N, size_t K, int format, void* out,
                            int dtype, size_t ldo, unsigned* status, void* stream) {
  if (!fp4_format_ok(format) || dtype_bytes((unsigned)dtype) == 0) return SSGD_ERR_ARG;
  if (!a_codes || !a_scales || !b_codes || !b_scales || !out || !status) return SSGD_ERR_NULL;
  if (M > SSGD_FP4_MAX_SIDE || N > SSGD_FP4_MAX_SIDE || K > SSGD_FP4_MAX_SIDE || ldo < N || mul_overflows(M, ldo) || mul_overflows(M * ldo, 4))
    return SSGD_ERR_SIZE;
  if (!aligned16(a_codes) || !aligned16(a_scales) || !aligned16(b_codes) || !aligned16(b_scales) ||
      reinterpret_cast<uintptr_t>(out) % dtype_bytes((unsigned)dtype) != 0 ||
      ((reinterpret_cast<uintptr_t>(a_tensor_scale) | reinterpret_cast<uintptr_t>(b_tensor_scale) | reinterpret_cast<uintptr_t>(status)) & 3u))
    return SSGD_ERR_ALIGN;
  if (M == 0 || N == 0) return SSGD_OK;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  if (format == SSGD_MXFP4)
    launch_matmul<SSGD_MXFP4>(a_codes, a_scales, a_tensor_scale, b_codes, b_scales, b_tensor_scale, M, N, K, out, dtype, ldo, s);
  else
    launch_matmul<SSGD_NVFP4>(a_codes, a_scales, a_tensor_scale, b_codes, b_scales, b_tensor_scale, M, N, K, out, dtype, ldo, s);
  return launch_status();
}

}  // extern "C"
