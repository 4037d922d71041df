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

// Largest magnitude of a matrix, as ordered bits (NaN above infinity); `out` starts at 0.  A maximum does not depend on
// the order, so the atomic gives the same bits every time.
template <typename T>
__device__ __forceinline__ unsigned piece_amax(const T* __restrict__ at, unsigned left, bool vec) {
  constexpr unsigned V = 16 / sizeof(T);
  unsigned top = 0;
  if (vec && left >= V) {
    const uint4 q = *reinterpret_cast<const uint4*>(at);
    const unsigned* w = reinterpret_cast<const unsigned*>(&q);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      top = max(top, magnitude_bits(low_to_float(T(), w[j])));
      if (sizeof(T) == 2) top = max(top, magnitude_bits(high_to_float(T(), w[j])));
    }
  } else {
    for (unsigned j = 0; j < V && j < left; ++j) top = max(top, magnitude_bits(to_float(at[j])));
  }
  return top;
}

// A CTA takes a rectangle of kAmaxRows rows by 256 pieces of 16 bytes, eight pieces of a thread in flight; rows that are
// not 16-byte aligned are read element by element, lanes side by side.
constexpr unsigned kAmaxRows = 8;
template <typename T>
__global__ void __launch_bounds__(kThreads)
fp4_amax_kernel(const T* __restrict__ x, unsigned rows, unsigned cols, size_t ldx, bool vec, unsigned tiles_c, unsigned* __restrict__ out) {
  constexpr unsigned V = 16 / sizeof(T), WIDE = kThreads * V;
  const unsigned r0 = blockIdx.x / tiles_c * kAmaxRows, c0 = blockIdx.x % tiles_c * WIDE;
  unsigned top = 0;
  if (vec) {
    const unsigned c = c0 + threadIdx.x * V;
#pragma unroll
    for (unsigned r = 0; r < kAmaxRows; ++r)
      if (r0 + r < rows && c < cols) top = max(top, piece_amax(x + (size_t)(r0 + r) * ldx + c, cols - c, true));
  } else {
#pragma unroll 2
    for (unsigned r = 0; r < kAmaxRows; ++r)
#pragma unroll
      for (unsigned q = 0; q < V; ++q) {
        const unsigned c = c0 + q * kThreads + threadIdx.x;
        if (r0 + r < rows && c < cols) top = max(top, magnitude_bits(to_float(x[(size_t)(r0 + r) * ldx + c])));
      }
  }
  top = __reduce_max_sync(0xFFFFFFFFu, top);
  __shared__ unsigned part[kThreads / 32];
  if ((threadIdx.x & 31u) == 0) part[threadIdx.x >> 5] = top;
  __syncthreads();
  if (threadIdx.x < 32) {
    const unsigned all = __reduce_max_sync(0xFFFFFFFFu, threadIdx.x < kThreads / 32 ? part[threadIdx.x] : 0u);
    if (threadIdx.x == 0) atomicMax(out, all);
  }
}

// Largest magnitude of a small matrix, by one CTA.
template <typename T>
__device__ __forceinline__ unsigned small_amax(const T* __restrict__ x, unsigned rows, unsigned cols, size_t ldx, bool vec) {
  constexpr unsigned V = 16 / sizeof(T);
  const unsigned pieces = (cols + V - 1) / V, total = rows * pieces;
  unsigned top = 0;
#pragma unroll 4
  for (unsigned i = threadIdx.x; i < total; i += kThreads) {
    const unsigned r = i / pieces, c = i % pieces * V;
    top = max(top, piece_amax(x + (size_t)r * ldx + c, cols - c, vec));
  }
  return top;
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

// Scale byte of a block from its largest magnitude, and what its values are divided by.
struct BlockScale {
  unsigned byte;
  float S;        // nv: block scale times tensor scale
  float inverse;  // nv: 1 / S to within the power of two correctly rounded; mx: 1 / S exactly
};
template <int FORMAT>
__device__ __forceinline__ BlockScale block_scale(unsigned top_bits, float tensor_scale, float tensor_inverse) {
  BlockScale b;
  b.S = 1.0f;
  if constexpr (FORMAT == SSGD_MXFP4) {
    // exponent of max|x| minus 2, kept at -127 or above (a block of zeros or subnormals)
    b.byte = top_bits >= 0x7F800000u ? 255u : (unsigned)max((int)(top_bits >> 23) - 2, 0);
    b.inverse = b.byte == 255u ? 1.0f : __uint_as_float((254u - b.byte) << 23);
  } else {
    const float s = __fdiv_rn(__fmul_rn(__uint_as_float(top_bits), tensor_inverse), 6.0f);
    const __nv_fp8_storage_t q = __nv_cvt_float_to_fp8(fminf(s, 448.0f), __NV_SATFINITE, __NV_E4M3);
    b.byte = top_bits >= 0x7F800000u ? 0x7Fu : max((unsigned)q, 1u);   // 1 = 2^-9, the least positive
    const float scale = b.byte == 0x7Fu ? 1.0f : e4m3_value(b.byte);
    b.S = scale * tensor_scale;
    b.inverse = __frcp_rn(scale) * tensor_inverse;
  }
  return b;
}

// The codes of one block (B / 8 words) and its scale byte.
template <int FORMAT, int B>
__device__ __forceinline__ unsigned quantise_block(float (&v)[B], float tensor_scale, float tensor_inverse, unsigned (&word)[B / 8]) {
  unsigned top = 0;
#pragma unroll
  for (int i = 0; i < B; ++i) top = max(top, magnitude_bits(v[i]));
  const BlockScale b = block_scale<FORMAT>(top, tensor_scale, tensor_inverse);
  if (FORMAT == SSGD_NVFP4 && __uint_as_float(top) * tensor_inverse > 1e30f) {   // a tensor scale far too small: saturate
    const float limit = 1e30f * tensor_scale;
#pragma unroll
    for (int i = 0; i < B; ++i) v[i] = fmaxf(-limit, fminf(limit, v[i]));
  }
#pragma unroll
  for (int i = 0; i < B; ++i) v[i] = FORMAT == SSGD_MXFP4 ? __fmul_rn(v[i], b.inverse) : quotient(v[i], b.S, b.inverse);
#pragma unroll
  for (int w = 0; w < B / 8; ++w) word[w] = top < 0x7F800000u ? fp4_pack8(v + 8 * w) : 0u;
  return b.byte;
}

// Elements of B * sizeof(T) bytes in 16-byte pieces as floats.
template <typename T, int B>
__device__ __forceinline__ void to_floats(const uint4 (&raw)[B * sizeof(T) / 16], float (&v)[B]) {
  const unsigned* w = reinterpret_cast<const unsigned*>(raw);
  if constexpr (sizeof(T) == 4) {
#pragma unroll
    for (int i = 0; i < B; ++i) v[i] = __uint_as_float(w[i]);
  } else {
#pragma unroll
    for (int i = 0; i < B / 2; ++i) {
      v[2 * i] = low_to_float(T(), w[i]);
      v[2 * i + 1] = high_to_float(T(), w[i]);
    }
  }
}

// A CTA takes a tile of 128 x 128: whole scale tiles and 64 bytes of codes of every row, in both directions.
//   rows     a thread takes a block of a row: its 16-byte loads are the tile's load, coalesced over the blocks of a row
//   columns  the tile goes through shared memory; lanes run along the columns (two 16-bit columns in a word), the codes
//            go back through shared memory so that 64 contiguous bytes of a column's row leave together
// Rows that are not 16-byte aligned are loaded element by element, coalesced, into the same shared tile.
constexpr unsigned kSide = 128;
constexpr unsigned kCodePitch = 80;                       // bytes of a column's 64 bytes of codes in shared memory

template <typename T> constexpr unsigned kTilePitch = kSide * sizeof(T) + 16;
template <typename T> unsigned tile_smem(bool tile, bool columns) {
  return (tile ? kSide * kTilePitch<T> : 0) + (columns ? kSide * kCodePitch : 0);
}
constexpr size_t kFusedAmax = 32768;                      // elements up to which every CTA finds the tensor's maximum itself

template <int FORMAT, bool ROWS, bool COLS, typename T>
__global__ void __launch_bounds__(kThreads)
fp4_quantise_kernel(const T* __restrict__ x, unsigned rows, unsigned cols, size_t ldx, bool vec, const float* __restrict__ amax,
                    float* __restrict__ tensor_scale, uint8_t* __restrict__ codes, uint8_t* __restrict__ scales,
                    uint8_t* __restrict__ codes_t, uint8_t* __restrict__ scales_t, unsigned tiles_c) {
  constexpr unsigned B = FORMAT == SSGD_MXFP4 ? 32 : 16, NB = kSide / B, ITEMS = kSide * NB / kThreads;
  constexpr unsigned PIECES = B * sizeof(T) / 16, PITCH = kTilePitch<T>;
  extern __shared__ __align__(16) unsigned char tile[];
  __shared__ __align__(16) uint8_t row_scales[NB * kSide], col_scales[COLS ? NB * kSide : 16];
  __shared__ unsigned part[kThreads / 32];
  pdl_launch_dependents();
  pdl_wait();
  const unsigned at = gridDim.x - 1 - blockIdx.x;         // from the end: what the maximum's pass read last is still in L2
  const unsigned r0 = at / tiles_c * kSide, c0 = at % tiles_c * kSide;

  uint4 raw[ITEMS][PIECES];
  if (vec) {
#pragma unroll
    for (unsigned u = 0; u < ITEMS; ++u) {
      const unsigned i = u * kThreads + threadIdx.x, row = r0 + i / NB, c = c0 + i % NB * B;
      const T* src = x + (size_t)row * ldx + c;
#pragma unroll
      for (unsigned q = 0; q < PIECES; ++q) {
        constexpr unsigned V = 16 / sizeof(T);
        raw[u][q] = make_uint4(0, 0, 0, 0);
        if (row < rows && c + (q + 1) * V <= cols) {
          raw[u][q] = *reinterpret_cast<const uint4*>(src + q * V);
        } else if (row < rows && c + q * V < cols) {      // the row ends inside this piece
          T e[V];
#pragma unroll
          for (unsigned j = 0; j < V; ++j) e[j] = c + q * V + j < cols ? src[q * V + j] : from_float<T>(0.0f);
          raw[u][q] = *reinterpret_cast<const uint4*>(e);
        }
      }
    }
  }
  float ts = 1.0f;
  if constexpr (FORMAT == SSGD_NVFP4) {
    float top;
    if (amax) {
      top = __ldg(amax);
    } else {
      const unsigned t = __reduce_max_sync(0xFFFFFFFFu, small_amax(x, rows, cols, ldx, vec));
      if ((threadIdx.x & 31u) == 0) part[threadIdx.x >> 5] = t;
      __syncthreads();
      unsigned all = 0;
#pragma unroll
      for (int w = 0; w < kThreads / 32; ++w) all = max(all, part[w]);
      top = __uint_as_float(all);
      if (blockIdx.x == 0 && threadIdx.x == 0) tensor_scale[1] = top;
    }
    ts = fp4_tensor_scale(top);
    if (blockIdx.x == 0 && threadIdx.x == 0) tensor_scale[0] = ts;
  }
  const float ti = __fdiv_rn(1.0f, ts);

  if (!vec) {
#pragma unroll 16
    for (unsigned i = threadIdx.x; i < kSide * kSide; i += kThreads) {
      const unsigned r = i / kSide, c = i % kSide;
      const bool in = r0 + r < rows && c0 + c < cols;
      *reinterpret_cast<T*>(tile + r * PITCH + c * sizeof(T)) = in ? x[(size_t)(r0 + r) * ldx + c0 + c] : from_float<T>(0.0f);
    }
    __syncthreads();
  }
  if (COLS || !vec) {
#pragma unroll
    for (unsigned u = 0; u < ITEMS; ++u) {
      const unsigned i = u * kThreads + threadIdx.x;
      uint4* slot = reinterpret_cast<uint4*>(tile + i / NB * PITCH + i % NB * B * sizeof(T));
#pragma unroll
      for (unsigned q = 0; q < PIECES; ++q) {
        if (vec) slot[q] = raw[u][q];
        else if (ROWS) raw[u][q] = slot[q];
      }
    }
  }
  if constexpr (ROWS) {
    const size_t row_bytes = (size_t)((cols + 31) / 32) * 16;
#pragma unroll
    for (unsigned u = 0; u < ITEMS; ++u) {
      const unsigned i = u * kThreads + threadIdx.x, r = i / NB, blk = i % NB, row = r0 + r, c = c0 + blk * B;
      float v[B];
      unsigned word[B / 8];
      to_floats<T, B>(raw[u], v);
      const unsigned byte = quantise_block<FORMAT, B>(v, ts, ti, word);
      row_scales[blk / 4 * 512 + (r & 31u) * 16 + (r >> 5) * 4 + (blk & 3u)] = row < rows && c < cols ? (uint8_t)byte : 0;
      if (row < rows && c < row_bytes * 2) {
        uint8_t* out = codes + (size_t)row * row_bytes + c / 2;
        if constexpr (B == 16) *reinterpret_cast<uint2*>(out) = make_uint2(word[0], word[1]);
        else *reinterpret_cast<uint4*>(out) = make_uint4(word[0], word[1], word[2], word[3]);
      }
    }
  }
  if (COLS) __syncthreads();
  if constexpr (COLS) {
    constexpr unsigned PAIR = sizeof(T) == 4 ? 1 : 2, WORDS = kSide / PAIR;     // columns of a word, words of a row
    unsigned char* out_codes = tile + kSide * PITCH;
#pragma unroll
    for (unsigned u = 0; u < WORDS * NB / kThreads; ++u) {
      const unsigned i = u * kThreads + threadIdx.x, w = i % WORDS, blk = i / WORDS;
      unsigned element[B];
#pragma unroll
      for (unsigned q = 0; q < B; ++q) element[q] = *reinterpret_cast<const unsigned*>(tile + (blk * B + q) * PITCH + w * 4);
#pragma unroll
      for (unsigned h = 0; h < PAIR; ++h) {
        float v[B];
        unsigned word[B / 8];
#pragma unroll
        for (unsigned q = 0; q < B; ++q)
          v[q] = PAIR == 1 ? __uint_as_float(element[q]) : h == 0 ? low_to_float(T(), element[q]) : high_to_float(T(), element[q]);
        const unsigned byte = quantise_block<FORMAT, B>(v, ts, ti, word), c = w * PAIR + h;
        col_scales[blk / 4 * 512 + (c & 31u) * 16 + (c >> 5) * 4 + (blk & 3u)] = c0 + c < cols && r0 + blk * B < rows ? (uint8_t)byte : 0;
        unsigned* out = reinterpret_cast<unsigned*>(out_codes + c * kCodePitch + blk * (B / 2));
        if constexpr (B == 16) *reinterpret_cast<uint2*>(out) = make_uint2(word[0], word[1]);
        else *reinterpret_cast<uint4*>(out) = make_uint4(word[0], word[1], word[2], word[3]);
      }
    }
  }
  __syncthreads();
  if constexpr (ROWS) {
    const size_t tiles_k = ((cols + B - 1) / B + 3) / 4, first = c0 / B / 4;
    if (threadIdx.x < NB / 4 * 32 && first + threadIdx.x / 32 < tiles_k)
      reinterpret_cast<uint4*>(scales + (r0 / kSide * tiles_k + first) * 512)[threadIdx.x] = reinterpret_cast<const uint4*>(row_scales)[threadIdx.x];
  }
  if constexpr (COLS) {
    const size_t row_bytes = (size_t)((rows + 31) / 32) * 16, tiles_k = ((rows + B - 1) / B + 3) / 4, first = r0 / B / 4;
    if (threadIdx.x < NB / 4 * 32 && first + threadIdx.x / 32 < tiles_k)
      reinterpret_cast<uint4*>(scales_t + (c0 / kSide * tiles_k + first) * 512)[threadIdx.x] = reinterpret_cast<const uint4*>(col_scales)[threadIdx.x];
#pragma unroll
    for (unsigned i = threadIdx.x; i < kSide * 4; i += kThreads) {
      const unsigned c = i / 4, b = i % 4 * 16;
      if (c0 + c < cols && r0 / 2 + b < row_bytes)
        *reinterpret_cast<uint4*>(codes_t + (size_t)(c0 + c) * row_bytes + r0 / 2 + b) = *reinterpret_cast<const uint4*>(tile + kSide * PITCH + c * kCodePitch + b);
    }
  }
}

// Eight values per thread and group, at places where the stores are 16-byte aligned: row by row the first group starts up
// to seven columns before the row, and a group's codes are cut out of two words.  A CTA takes kGroups x 256 groups from
// its place in the sequence of all rows' groups; the one 64-bit division is the CTA's.
constexpr unsigned kGroups = 4;

template <int FORMAT, typename T>
__global__ void __launch_bounds__(kThreads)
fp4_dequantise_kernel(const uint8_t* __restrict__ codes, const uint8_t* __restrict__ scales, const float* __restrict__ tensor_scale,
                      unsigned rows, unsigned cols, T* __restrict__ out, size_t ldo, unsigned groups) {
  constexpr unsigned B = FORMAT == SSGD_MXFP4 ? 32 : 16, V = 16 / sizeof(T);
  __shared__ unsigned start[2];
  if (threadIdx.x == 0) {
    const size_t first = (size_t)blockIdx.x * (kThreads * kGroups);
    start[0] = (unsigned)(first / groups);
    start[1] = (unsigned)(first % groups);
  }
  __syncthreads();
  pdl_launch_dependents();
  pdl_wait();
  const float ts = FORMAT == SSGD_NVFP4 && tensor_scale ? __ldg(tensor_scale) : 1.0f;
  const unsigned row_words = (cols + 31) / 32 * 4;
  const size_t tiles_k = ((cols + B - 1) / B + 3) / 4;
  T* line[kGroups];
  int column[kGroups];
  unsigned lo[kGroups], hi[kGroups], byte0[kGroups], byte1[kGroups];
#pragma unroll
  for (unsigned u = 0; u < kGroups; ++u) {
    const unsigned from = start[1] + u * kThreads + threadIdx.x, row = start[0] + from / groups;
    line[u] = out + (size_t)row * ldo;
    const unsigned back = (unsigned)(reinterpret_cast<uintptr_t>(line[u]) / sizeof(T)) & (V - 1);   // columns before the row that complete 16 bytes
    const int c = (int)(from % groups * 8) - (int)back;                                              // first column of the group
    column[u] = row < rows ? c : (int)cols;
    lo[u] = hi[u] = byte0[u] = byte1[u] = 0;
    if (row < rows && c < (int)cols) {
      const uint32_t* words = reinterpret_cast<const uint32_t*>(codes) + (size_t)row * row_words;
      const int w = c >> 3;                                                                          // rounds down
      if (w >= 0) lo[u] = words[w];
      if (((unsigned)c & 7u) && (unsigned)(w + 1) < row_words) hi[u] = words[w + 1];
      const unsigned b0 = (unsigned)max(c, 0) / B, b1 = min((unsigned)(c + 7), cols - 1) / B;
      byte0[u] = scales[fp4_scale_index(row, b0, tiles_k)];
      byte1[u] = b1 == b0 ? byte0[u] : scales[fp4_scale_index(row, b1, tiles_k)];
    }
  }
#pragma unroll
  for (unsigned u = 0; u < kGroups; ++u) {
    const int c = column[u];
    if (c >= (int)cols) continue;
    const unsigned eight = __funnelshift_r(lo[u], hi[u], ((unsigned)c & 7u) * 4);
    const float s0 = __fmul_rn(fp4_scale_value<FORMAT>(byte0[u]), ts), s1 = __fmul_rn(fp4_scale_value<FORMAT>(byte1[u]), ts);
    const int change = (max(c, 0) / (int)B + 1) * (int)B - c;           // the group's place from which the second scale holds
    float v[8];
#pragma unroll
    for (int j = 0; j < 8; j += 2) {
      const float2 two = fp4_pair_value(eight >> (4 * j));
      v[j] = __fmul_rn(two.x, j < change ? s0 : s1);
      v[j + 1] = __fmul_rn(two.y, j + 1 < change ? s0 : s1);
    }
    T* o = line[u] + c;
    if (c >= 0 && c + 8 <= (int)cols) {
      if constexpr (sizeof(T) == 4) {
        store4(o, make_float4(v[0], v[1], v[2], v[3]));
        store4(o + 4, make_float4(v[4], v[5], v[6], v[7]));
      } else {
        __stcs(reinterpret_cast<uint4*>(o), make_uint4(pack2(T(), v[0], v[1]), pack2(T(), v[2], v[3]), pack2(T(), v[4], v[5]), pack2(T(), v[6], v[7])));
      }
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j)
        if (c + j >= 0 && c + j < (int)cols) o[j] = from_float<T>(v[j]);
    }
  }
}

template <typename T>
bool rows_aligned(const T* x, size_t ldx) { return aligned16(x) && ldx * sizeof(T) % 16 == 0; }

template <int FORMAT, bool ROWS, bool COLS, typename T>
ssgd_status launch_quantise(const T* x, size_t rows, size_t cols, size_t ldx, const float* amax, float* tensor_scale, uint8_t* codes,
                            uint8_t* scales, uint8_t* codes_t, uint8_t* scales_t, cudaStream_t s) {
  const size_t tiles_c = (cols + kSide - 1) / kSide, tiles = (rows + kSide - 1) / kSide * tiles_c;
  if (tiles > kMaxGrid) return SSGD_ERR_SIZE;
  const bool vec = rows_aligned(x, ldx);
  const unsigned smem = tile_smem<T>(COLS || !vec, COLS);
  auto kernel = fp4_quantise_kernel<FORMAT, ROWS, COLS, T>;
  static unsigned long long seen = 0;
  if (smem > 32768 && !allow_smem(reinterpret_cast<const void*>(kernel), tile_smem<T>(true, COLS), &seen)) return SSGD_ERR_CUDA;
  launch_kernel(kernel, dim3((unsigned)tiles), dim3(kThreads), smem, s, true, x, (unsigned)rows, (unsigned)cols, ldx, vec, amax, tensor_scale,
                codes, scales, codes_t, scales_t, (unsigned)tiles_c);
  return launch_status();
}

template <int FORMAT, typename T>
ssgd_status quantise_typed(const T* x, size_t rows, size_t cols, size_t ldx, const float* amax, float* tensor_scale, uint8_t* codes,
                           uint8_t* scales, uint8_t* codes_t, uint8_t* scales_t, cudaStream_t s) {
  if (FORMAT == SSGD_NVFP4 && !amax && rows * cols > kFusedAmax) {
    if (cudaMemsetAsync(tensor_scale + 1, 0, sizeof(float), s) != cudaSuccess) return SSGD_ERR_CUDA;
    const size_t wide = kThreads * 16 / sizeof(T), tiles_c = (cols + wide - 1) / wide, ctas = (rows + kAmaxRows - 1) / kAmaxRows * tiles_c;
    if (ctas > kMaxGrid) return SSGD_ERR_SIZE;
    fp4_amax_kernel<<<(unsigned)ctas, kThreads, 0, s>>>(x, (unsigned)rows, (unsigned)cols, ldx, rows_aligned(x, ldx), (unsigned)tiles_c,
                                                        reinterpret_cast<unsigned*>(tensor_scale + 1));
    amax = tensor_scale + 1;
  }
  if (codes && codes_t) return launch_quantise<FORMAT, true, true>(x, rows, cols, ldx, amax, tensor_scale, codes, scales, codes_t, scales_t, s);
  if (codes) return launch_quantise<FORMAT, true, false>(x, rows, cols, ldx, amax, tensor_scale, codes, scales, codes_t, scales_t, s);
  return launch_quantise<FORMAT, false, true>(x, rows, cols, ldx, amax, tensor_scale, codes, scales, codes_t, scales_t, s);
}

template <typename T>
ssgd_status quantise_format(const T* x, size_t rows, size_t cols, size_t ldx, int format, const float* amax, float* tensor_scale, uint8_t* codes,
                            uint8_t* scales, uint8_t* codes_t, uint8_t* scales_t, cudaStream_t s) {
  return format == SSGD_MXFP4 ? quantise_typed<SSGD_MXFP4>(x, rows, cols, ldx, amax, tensor_scale, codes, scales, codes_t, scales_t, s)
                              : quantise_typed<SSGD_NVFP4>(x, rows, cols, ldx, amax, tensor_scale, codes, scales, codes_t, scales_t, s);
}

template <int FORMAT, typename T>
ssgd_status launch_dequantise(const uint8_t* codes, const uint8_t* scales, const float* ts, size_t rows, size_t cols, T* out, size_t ldo, cudaStream_t s) {
  const size_t groups = (cols + 7) / 8 + (rows_aligned(out, rows > 1 ? ldo : 16 / sizeof(T)) ? 0 : 1), ctas = (rows * groups + kThreads * kGroups - 1) / (kThreads * kGroups);
  if (ctas > kMaxGrid) return SSGD_ERR_SIZE;
  launch_kernel(fp4_dequantise_kernel<FORMAT, T>, dim3((unsigned)ctas), dim3(kThreads), 0, s, true, codes, scales, ts, (unsigned)rows, (unsigned)cols,
                out, ldo, (unsigned)groups);
  return launch_status();
}

template <typename T>
ssgd_status dequantise_format(const uint8_t* codes, const uint8_t* scales, const float* ts, int format, size_t rows, size_t cols, T* out, size_t ldo,
                              cudaStream_t s) {
  return format == SSGD_MXFP4 ? launch_dequantise<SSGD_MXFP4>(codes, scales, ts, rows, cols, out, ldo, s)
                              : launch_dequantise<SSGD_NVFP4>(codes, scales, ts, rows, cols, out, ldo, s);
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
    case SSGD_F32: return quantise_format(static_cast<const float*>(x), rows, cols, ldx, format, amax, tensor_scale, codes, scales, codes_t, scales_t, s);
    case SSGD_BF16: return quantise_format(static_cast<const __nv_bfloat16*>(x), rows, cols, ldx, format, amax, tensor_scale, codes, scales, codes_t, scales_t, s);
    default: return quantise_format(static_cast<const __half*>(x), rows, cols, ldx, format, amax, tensor_scale, codes, scales, codes_t, scales_t, s);
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
  switch (dtype) {
    case SSGD_F32: return dequantise_format(codes, scales, tensor_scale, format, rows, cols, static_cast<float*>(out), ldo, s);
    case SSGD_BF16: return dequantise_format(codes, scales, tensor_scale, format, rows, cols, static_cast<__nv_bfloat16*>(out), ldo, s);
    default: return dequantise_format(codes, scales, tensor_scale, format, rows, cols, static_cast<__half*>(out), ldo, s);
  }
}

}  // extern "C"
