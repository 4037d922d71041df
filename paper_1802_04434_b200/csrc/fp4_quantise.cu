// Quantisation to microscaled 4-bit numbers, by rows and by columns, and its inverse.  See include/signsgd.h.
//
//   mx: S = 2^(floor(log2 max|x|) - 2) over a block;   nv: S = max(e4m3(max|x| / t / 6), 2^-9) * t, t the tensor scale
//   code = nearest 4-bit value to x / S, ties to the even code, magnitudes above 6 to 6
// A block that holds an infinity or a NaN gets the NaN scale: it reads back as NaN, and so do products with it.

#include "host_calls.h"
#include "dtypes.cuh"
#include "fp4.cuh"

namespace {

__device__ __forceinline__ unsigned magnitude_bits(float v) { return __float_as_uint(v) & 0x7FFFFFFFu; }

// Larger magnitude of two words of elements (one fp32 or two 16-bit), a NaN carried through; the sign is not defined.
__device__ __forceinline__ unsigned larger(float, unsigned a, unsigned b) {
  unsigned r;
  asm("{\n\t.reg .f32 x, y;\n\tmov.b32 x, %1;\n\tmov.b32 y, %2;\n\tmax.NaN.xorsign.abs.f32 x, x, y;\n\tmov.b32 %0, x;\n\t}" : "=r"(r) : "r"(a), "r"(b));
  return r;
}
__device__ __forceinline__ unsigned larger(__nv_bfloat16, unsigned a, unsigned b) {
  unsigned r;
  asm("max.NaN.xorsign.abs.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
  return r;
}
__device__ __forceinline__ unsigned larger(__half, unsigned a, unsigned b) {
  unsigned r;
  asm("max.NaN.xorsign.abs.f16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
  return r;
}

// Largest magnitude of an fp32 or of both 16-bit elements of a word, as the bits of a float.
template <typename T> __device__ __forceinline__ unsigned top_of_word(unsigned w) {
  const unsigned lo = magnitude_bits(low_to_float(T(), w));
  return sizeof(T) == 4 ? lo : max(lo, magnitude_bits(high_to_float(T(), w)));
}

// One element as a word of elements.
__device__ __forceinline__ unsigned word_of(float v) { return __float_as_uint(v); }
__device__ __forceinline__ unsigned word_of(__nv_bfloat16 v) { return __bfloat16_as_ushort(v); }
__device__ __forceinline__ unsigned word_of(__half v) { return __half_as_ushort(v); }

// Two fp32 operations in one instruction.
__device__ __forceinline__ uint64_t pair_of(float lo, float hi) {
  uint64_t r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(lo), "f"(hi));
  return r;
}
__device__ __forceinline__ uint64_t mul_pair(uint64_t a, uint64_t b) {
  uint64_t r;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ uint64_t fma_pair(uint64_t a, uint64_t b, uint64_t c) {
  uint64_t r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
  return r;
}

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

// Largest magnitude of what each CTA sees, as bits, to a place of its own: no memory has to start at zero, and every CTA
// of the quantisation that follows takes the largest of them.  A CTA takes rectangles: `wide` threads (a power of two) lie
// along a row, a piece of 16 bytes each, the others in rows below, every thread ROWS rows, all in flight.  Rows that are not
// 16-byte aligned are read element by element, lanes side by side: which of the two is the matrix's, not a thread's, choice,
// because the lanes' elements lie elsewhere than their pieces.
constexpr unsigned kAmaxThreads = 512, kAmaxCtas = 2;     // CTAs of an SM
template <unsigned ROWS, typename T>
__global__ void __launch_bounds__(kAmaxThreads, kAmaxCtas)
fp4_amax_kernel(const T* __restrict__ x, unsigned rows, unsigned cols, size_t ldx, bool vec, unsigned wide, unsigned strips, unsigned long long units,
                unsigned* __restrict__ out) {
  constexpr unsigned V = 16 / sizeof(T);
  pdl_launch_dependents();
  pdl_wait();
  const unsigned lane = threadIdx.x & (wide - 1), below = threadIdx.x / wide, high = kAmaxThreads / wide;
  unsigned w = 0;
  for (unsigned long long i = blockIdx.x; i < units; i += gridDim.x) {
    const unsigned r0 = (unsigned)(i / strips) * (high * ROWS) + below, c0 = (unsigned)(i % strips) * (wide * V);
    const unsigned c = c0 + lane * V;
    if (vec) {
      if (r0 + (ROWS - 1) * high < rows && c + V <= cols) {
        uint4 q[ROWS];
#pragma unroll
        for (unsigned r = 0; r < ROWS; ++r) q[r] = *reinterpret_cast<const uint4*>(x + (size_t)(r0 + r * high) * ldx + c);
#pragma unroll
        for (unsigned r = 0; r < ROWS; ++r) w = larger(T(), larger(T(), w, larger(T(), q[r].x, q[r].y)), larger(T(), q[r].z, q[r].w));
      } else if (c < cols) {                              // the matrix ends within the thread's rows or its piece
        const unsigned left = min(V, cols - c);
#pragma unroll (ROWS < 4 ? ROWS : 4)
        for (unsigned r = 0; r < ROWS; ++r)
#pragma unroll
          for (unsigned e = 0; e < V; ++e)
            if (r0 + r * high < rows && e < left) w = larger(T(), w, word_of(x[(size_t)(r0 + r * high) * ldx + c + e]));
      }
    } else {
#pragma unroll (ROWS < 4 ? ROWS : 4)
      for (unsigned r = 0; r < ROWS; ++r)
#pragma unroll
        for (unsigned q = 0; q < V; ++q) {
          const unsigned e = c0 + q * wide + lane;
          if (r0 + r * high < rows && e < cols) w = larger(T(), w, word_of(x[(size_t)(r0 + r * high) * ldx + e]));
        }
    }
  }
  const unsigned top = __reduce_max_sync(0xFFFFFFFFu, top_of_word<T>(w));
  __shared__ unsigned part[kAmaxThreads / 32];
  if ((threadIdx.x & 31u) == 0) part[threadIdx.x >> 5] = top;
  __syncthreads();
  if (threadIdx.x < 32) {
    const unsigned all = __reduce_max_sync(0xFFFFFFFFu, threadIdx.x < kAmaxThreads / 32 ? part[threadIdx.x] : 0u);
    if (threadIdx.x == 0) out[blockIdx.x] = all;
  }
}

// Largest magnitude of a small matrix, by one CTA.
template <unsigned THREADS, typename T>
__device__ __forceinline__ unsigned small_amax(const T* __restrict__ x, unsigned rows, unsigned cols, size_t ldx, bool vec) {
  constexpr unsigned V = 16 / sizeof(T);
  const unsigned pieces = (cols + V - 1) / V, total = rows * pieces;
  unsigned top = 0;
#pragma unroll 4
  for (unsigned i = threadIdx.x; i < total; i += THREADS) {
    const unsigned r = i / pieces, c = i % pieces * V;
    top = max(top, piece_amax(x + (size_t)r * ldx + c, cols - c, vec));
  }
  return top;
}

// Eight values (four pairs) to the four bytes of their codes: nearest, ties to even, saturating.
__device__ __forceinline__ unsigned fp4_pack8(const uint64_t (&v)[4]) {
  unsigned out;
  asm("{\n\t.reg .b8 b0, b1, b2, b3;\n\t.reg .f32 l0, l1, l2, l3, h0, h1, h2, h3;\n\t"
      "mov.b64 {l0, h0}, %1;\n\tmov.b64 {l1, h1}, %2;\n\tmov.b64 {l2, h2}, %3;\n\tmov.b64 {l3, h3}, %4;\n\t"
      "cvt.rn.satfinite.e2m1x2.f32 b0, h0, l0;\n\t"
      "cvt.rn.satfinite.e2m1x2.f32 b1, h1, l1;\n\t"
      "cvt.rn.satfinite.e2m1x2.f32 b2, h2, l2;\n\t"
      "cvt.rn.satfinite.e2m1x2.f32 b3, h3, l3;\n\t"
      "mov.b32 %0, {b0, b1, b2, b3};\n\t}"
      : "=r"(out)
      : "l"(v[0]), "l"(v[1]), "l"(v[2]), "l"(v[3]));
  return out;
}

// How a block is divided by its scale S: mx multiplies by 1 / S, a power of two.  nv multiplies by a reciprocal in two parts,
// high <= 1 / S and low >= 0, as fma(x, high, x * low): off by 2^-43 before the one rounding, so the quotient is the correctly
// rounded one except within that of halfway, and a tie between two codes stays a tie (a single fp32 reciprocal would send 1 %
// of a bf16 tensor's values to the wrong side).  Two multiplications instead of a division's ten instructions.  A quotient
// beyond fp32 (a tensor scale far too small) becomes an infinity of x's sign, and that saturates.
struct BlockScale {
  unsigned byte;
  float high, low;
  bool finite;
};
template <int FORMAT>
__device__ __forceinline__ BlockScale block_scale(unsigned top_bits, float tensor_inverse) {
  BlockScale b;
  b.finite = top_bits < 0x7F800000u;
  b.low = 0.0f;
  if constexpr (FORMAT == SSGD_MXFP4) {
    // exponent of max|x| minus 2, kept at -127 or above (a block of zeros or subnormals)
    b.byte = b.finite ? (unsigned)max((int)(top_bits >> 23) - 2, 0) : 255u;
    b.high = __uint_as_float((254u - b.byte) << 23);                    // not used where byte is 255
  } else {
    // max|x| / t / 6 with 1 / 6 in two parts, then to the nearest E4M3 number, at most 448
    const float v = __fmul_rn(__uint_as_float(top_bits), tensor_inverse);
    const float s = __fmaf_rn(v, 0x1.555554p-3f, __fmul_rn(v, 0x1.555556p-27f));
    unsigned short q;
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(q) : "f"(0.0f), "f"(s));
    const unsigned byte = max((unsigned)q, 1u);                         // 1 = 2^-9, the least positive
    unsigned half2;
    asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(half2) : "h"((unsigned short)byte));
    const float scale = __low2float(*reinterpret_cast<const __half2*>(&half2));
    float r;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(scale));
    r = __fmul_rn(r, 1.0f - 0x1p-22f);                                  // below 1 / scale for certain
    b.high = r * tensor_inverse;
    b.low = __fmul_rn(__fmaf_rn(-scale, r, 1.0f), b.high);
    b.byte = b.finite ? byte : 0x7Fu;
  }
  return b;
}

// The codes of one block of B values, given as pairs, and its scale byte.
template <int FORMAT, int B>
__device__ __forceinline__ unsigned quantise_block(uint64_t (&v)[B / 2], unsigned top_bits, float tensor_inverse, unsigned (&word)[B / 8]) {
  const BlockScale b = block_scale<FORMAT>(top_bits, tensor_inverse);
  const uint64_t high = pair_of(b.high, b.high), low = pair_of(b.low, b.low);
#pragma unroll
  for (int i = 0; i < B / 2; ++i) v[i] = FORMAT == SSGD_MXFP4 ? mul_pair(v[i], high) : fma_pair(v[i], high, mul_pair(v[i], low));
#pragma unroll
  for (int w = 0; w < B / 8; ++w) {
    const uint64_t four[4] = {v[4 * w], v[4 * w + 1], v[4 * w + 2], v[4 * w + 3]};
    word[w] = b.finite ? fp4_pack8(four) : 0u;
  }
  return b.byte;
}

// A block that lies along words of elements.
template <int FORMAT, int B, typename T>
__device__ __forceinline__ unsigned quantise_words(const unsigned* w, float tensor_inverse, unsigned (&word)[B / 8]) {
  constexpr int W = B * (int)sizeof(T) / 4;
  unsigned top = w[0];
#pragma unroll
  for (int i = 1; i < W; ++i) top = larger(T(), top, w[i]);
  uint64_t v[B / 2];
#pragma unroll
  for (int i = 0; i < B / 2; ++i)
    v[i] = sizeof(T) == 4 ? pair_of(__uint_as_float(w[(2 * i) % W]), __uint_as_float(w[(2 * i + 1) % W])) : pair_of(low_to_float(T(), w[i]), high_to_float(T(), w[i]));
  return quantise_block<FORMAT, B>(v, top_of_word<T>(top), tensor_inverse, word);
}

// A CTA takes a tile of 128 x 128: whole scale tiles and 64 bytes of codes of every row, in both directions.  The tile goes
// to shared memory by asynchronous copies, lanes side by side, in pieces of 16 bytes where the rows allow it, else of 4,
// else element by element through registers; what lies outside the matrix becomes 0.
//   rows     lanes run down the rows (a row is 16 bytes longer than its elements: no bank conflicts), a thread takes a
//            block of a row
//   columns  lanes run along the columns (two 16-bit columns in a word), a thread takes a block of a column, or of two
// Either way the codes go back through shared memory, so that 64 contiguous bytes of a row of codes leave together.
constexpr unsigned kSide = 128;
constexpr unsigned kCodePitch = 72;                       // of the 64 bytes of codes of a row in shared memory
template <typename T> constexpr unsigned kTilePitch = kSide * sizeof(T) + 16;
template <typename T> constexpr unsigned kTileSmem = kSide * kTilePitch<T> + kSide * kCodePitch;
constexpr size_t kFusedAmax = SSGD_FP4_SMALL;             // elements up to which every CTA finds the tensor's maximum itself

template <unsigned BYTES>
__device__ __forceinline__ void copy_async(unsigned dst, const void* src, unsigned valid) {   // `valid` bytes, the rest 0
  asm volatile("cp.async.ca.shared.global [%0], [%1], %2, %3;" ::"r"(dst), "l"(src), "n"(BYTES), "r"(valid) : "memory");
}

template <unsigned BYTES, unsigned THREADS, typename T>
__device__ __forceinline__ void load_tile(unsigned tile, const T* __restrict__ x, unsigned rows, unsigned cols, size_t ldx, unsigned r0, unsigned c0) {
  constexpr unsigned V = BYTES / sizeof(T), PER_ROW = kSide / V;
#pragma unroll 8
  for (unsigned i = threadIdx.x; i < kSide * PER_ROW; i += THREADS) {
    const unsigned r = i / PER_ROW, c = i % PER_ROW * V;
    const bool in = r0 + r < rows && c0 + c < cols;
    const unsigned valid = in ? min(V, cols - (c0 + c)) * (unsigned)sizeof(T) : 0u;
    copy_async<BYTES>(tile + r * kTilePitch<T> + c * (unsigned)sizeof(T), in ? x + (size_t)(r0 + r) * ldx + c0 + c : x, valid);
  }
}

// The scale tiles of a tile of rows, from shared memory.
template <unsigned NB>
__device__ __forceinline__ void write_scales(const uint8_t* staged_scales, uint8_t* __restrict__ scales, unsigned cols, unsigned r0, unsigned c0) {
  constexpr unsigned B = kSide / NB;
  const size_t tiles_k = ((cols + B - 1) / B + 3) / 4, first = c0 / B / 4;
  if (threadIdx.x < NB / 4 * 32 && first + threadIdx.x / 32 < tiles_k)
    reinterpret_cast<uint4*>(scales + (r0 / kSide * tiles_k + first) * 512)[threadIdx.x] = reinterpret_cast<const uint4*>(staged_scales)[threadIdx.x];
}

// 64 bytes of codes of each of the tile's rows, and its scale tiles, from shared memory.
template <unsigned NB, unsigned THREADS>
__device__ __forceinline__ void write_out(const unsigned char* staged, const uint8_t* staged_scales, uint8_t* __restrict__ codes, uint8_t* __restrict__ scales,
                                          unsigned rows, unsigned cols, unsigned r0, unsigned c0) {
  const size_t row_bytes = (size_t)((cols + 31) / 32) * 16;
#pragma unroll
  for (unsigned i = threadIdx.x; i < kSide * 4; i += THREADS) {
    const unsigned r = i / 4, at = i % 4 * 16;
    if (r0 + r < rows && c0 / 2 + at < row_bytes) {
      const uint2 lo = *reinterpret_cast<const uint2*>(staged + r * kCodePitch + at), hi = *reinterpret_cast<const uint2*>(staged + r * kCodePitch + at + 8);
      *reinterpret_cast<uint4*>(codes + (size_t)(r0 + r) * row_bytes + c0 / 2 + at) = make_uint4(lo.x, lo.y, hi.x, hi.y);
    }
  }
  write_scales<NB>(staged_scales, scales, cols, r0, c0);
}

template <int B>
__device__ __forceinline__ void stage_codes(unsigned char* to, const unsigned (&word)[B / 8]) {
#pragma unroll
  for (int i = 0; i < B / 16; ++i) *reinterpret_cast<uint2*>(to + 8 * i) = make_uint2(word[2 * i], word[2 * i + 1]);
}

// The tensor scale (1 for mx), from the caller's maximum, from the maxima of the pass before, or from a small matrix itself;
// the first CTA writes down what was found.  Every thread of the CTA must call.
template <int FORMAT, unsigned THREADS, typename T>
__device__ __forceinline__ float tensor_scale_of(const T* __restrict__ x, unsigned rows, unsigned cols, size_t ldx, bool vec, const float* __restrict__ amax,
                                                 unsigned maxima, float* tensor_scale, unsigned* part) {
  if constexpr (FORMAT == SSGD_MXFP4) return 1.0f;
  float top;
  if (amax) {
    top = __ldg(amax);
  } else if (maxima > 0) {                                // every warp for itself
    unsigned t = 0;
    for (unsigned i = threadIdx.x & 31u; i < maxima; i += 32) t = max(t, __float_as_uint(tensor_scale[2 + i]));
    top = __uint_as_float(__reduce_max_sync(0xFFFFFFFFu, t));
  } else {
    const unsigned t = __reduce_max_sync(0xFFFFFFFFu, small_amax<THREADS>(x, rows, cols, ldx, vec));
    if ((threadIdx.x & 31u) == 0) part[threadIdx.x >> 5] = t;
    __syncthreads();
    unsigned all = 0;
#pragma unroll
    for (unsigned w = 0; w < THREADS / 32; ++w) all = max(all, part[w]);
    top = __uint_as_float(all);
  }
  const float ts = fp4_tensor_scale(top);
  if (blockIdx.x == 0 && threadIdx.x == 0) {
    tensor_scale[0] = ts;
    if (!amax) tensor_scale[1] = top;
  }
  return ts;
}

// piece: bytes that a copy of x's elements may have (16, 4, or 0: none, its rows start at odd 16-bit elements)
template <int FORMAT, bool ROWS, bool COLS, unsigned THREADS, typename T>
__global__ void __launch_bounds__(THREADS, THREADS == 512 ? 1 : 0)
fp4_quantise_kernel(const T* __restrict__ x, unsigned rows, unsigned cols, size_t ldx, unsigned piece, const float* __restrict__ amax,
                    unsigned maxima, float* tensor_scale, uint8_t* __restrict__ codes, uint8_t* __restrict__ scales,
                    uint8_t* __restrict__ codes_t, uint8_t* __restrict__ scales_t, unsigned tiles_c) {
  constexpr unsigned B = FORMAT == SSGD_MXFP4 ? 32 : 16, NB = kSide / B;
  constexpr unsigned PIECES = B * sizeof(T) / 16, PITCH = kTilePitch<T>;
  extern __shared__ __align__(16) unsigned char tile[];
  __shared__ __align__(16) uint8_t staged_scales[NB * kSide];
  __shared__ unsigned part[THREADS / 32];
  unsigned char* staged = tile + kSide * PITCH;
  pdl_launch_dependents();
  pdl_wait();
  const unsigned at = gridDim.x - 1 - blockIdx.x;         // from the end: what the maximum's pass read last is still in L2
  const unsigned r0 = at / tiles_c * kSide, c0 = at % tiles_c * kSide;

  if (piece == 16) {
    load_tile<16, THREADS>((unsigned)__cvta_generic_to_shared(tile), x, rows, cols, ldx, r0, c0);
  } else if (sizeof(T) == 4 || piece == 4) {
    load_tile<4, THREADS>((unsigned)__cvta_generic_to_shared(tile), x, rows, cols, ldx, r0, c0);
  } else {
#pragma unroll 16
    for (unsigned i = threadIdx.x; i < kSide * kSide; i += THREADS) {
      const unsigned r = i / kSide, c = i % kSide;
      const bool in = r0 + r < rows && c0 + c < cols;
      *reinterpret_cast<T*>(tile + r * PITCH + c * sizeof(T)) = in ? x[(size_t)(r0 + r) * ldx + c0 + c] : from_float<T>(0.0f);
    }
  }
  const float ti = __fdiv_rn(1.0f, tensor_scale_of<FORMAT, THREADS>(x, rows, cols, ldx, piece == 16, amax, maxima, tensor_scale, part));
  asm volatile("cp.async.wait_all;" ::: "memory");
  __syncthreads();

  if constexpr (ROWS) {
#pragma unroll
    for (unsigned u = 0; u < (kSide * NB + THREADS - 1) / THREADS; ++u) {
      const unsigned i = u * THREADS + threadIdx.x, r = i % kSide, blk = i / kSide;
      uint4 raw[PIECES];
#pragma unroll
      for (unsigned q = 0; q < PIECES; ++q) raw[q] = *reinterpret_cast<const uint4*>(tile + r * PITCH + blk * B * sizeof(T) + q * 16);
      unsigned word[B / 8];
      const unsigned byte = quantise_words<FORMAT, B, T>(reinterpret_cast<const unsigned*>(raw), ti, word);
      staged_scales[blk / 4 * 512 + (r & 31u) * 16 + (r >> 5) * 4 + (blk & 3u)] = r0 + r < rows && c0 + blk * B < cols ? (uint8_t)byte : 0;
      stage_codes<B>(staged + r * kCodePitch + blk * (B / 2), word);
    }
    __syncthreads();
    write_out<NB, THREADS>(staged, staged_scales, codes, scales, rows, cols, r0, c0);
    if (COLS) __syncthreads();
  }
  if constexpr (COLS) {
    constexpr unsigned PAIR = sizeof(T) == 4 ? 1 : 2, WORDS = kSide / PAIR;     // columns of a word, words of a row
#pragma unroll
    for (unsigned u = 0; u < (WORDS * NB + THREADS - 1) / THREADS; ++u) {
      const unsigned i = u * THREADS + threadIdx.x, w = i % WORDS, blk = i / WORDS;
      if (WORDS * NB % THREADS != 0 && i >= WORDS * NB) continue;
      unsigned element[B];
#pragma unroll
      for (unsigned q = 0; q < B; ++q) element[q] = *reinterpret_cast<const unsigned*>(tile + (blk * B + q) * PITCH + w * 4);
      unsigned top = element[0];
#pragma unroll
      for (unsigned q = 1; q < B; ++q) top = larger(T(), top, element[q]);
#pragma unroll
      for (unsigned h = 0; h < PAIR; ++h) {
        uint64_t v[B / 2];
        unsigned word[B / 8];
#pragma unroll
        for (unsigned q = 0; q < B / 2; ++q)
          v[q] = h == 0 ? pair_of(low_to_float(T(), element[2 * q]), low_to_float(T(), element[2 * q + 1]))
                        : pair_of(high_to_float(T(), element[2 * q]), high_to_float(T(), element[2 * q + 1]));
        const unsigned c = w * PAIR + h;
        const unsigned byte = quantise_block<FORMAT, B>(v, magnitude_bits(h == 0 ? low_to_float(T(), top) : high_to_float(T(), top)), ti, word);
        staged_scales[blk / 4 * 512 + (c & 31u) * 16 + (c >> 5) * 4 + (blk & 3u)] = c0 + c < cols && r0 + blk * B < rows ? (uint8_t)byte : 0;
        stage_codes<B>(staged + c * kCodePitch + blk * (B / 2), word);
      }
    }
    __syncthreads();
    write_out<NB, THREADS>(staged, staged_scales, codes_t, scales_t, cols, rows, c0, r0);
  }
}

// By rows only, 16-bit elements, rows at multiples of 16 bytes: the same tiles without the way through shared memory.  A thread
// loads its block (lanes over the blocks of a row, 16-byte pieces), and its codes leave with its neighbours', 64 bytes of a
// row (B200, 8192 x 8192 bf16, mx / nv: 27 / 29 us; through shared memory 35 / 39; fp32, mx: 65 instead of 52, so not for it).
template <int FORMAT, typename T>
__global__ void __launch_bounds__(kThreads)
fp4_quantise_rows_kernel(const T* __restrict__ x, unsigned rows, unsigned cols, size_t ldx, const float* __restrict__ amax, unsigned maxima,
                         float* tensor_scale, uint8_t* __restrict__ codes, uint8_t* __restrict__ scales, unsigned tiles_c) {
  constexpr unsigned B = FORMAT == SSGD_MXFP4 ? 32 : 16, NB = kSide / B, ITEMS = kSide * NB / kThreads, PIECES = B * sizeof(T) / 16, V = 16 / sizeof(T);
  __shared__ __align__(16) uint8_t staged_scales[NB * kSide];
  __shared__ unsigned part[kThreads / 32];
  pdl_launch_dependents();
  pdl_wait();
  const unsigned at = gridDim.x - 1 - blockIdx.x, r0 = at / tiles_c * kSide, c0 = at % tiles_c * kSide;
  uint4 raw[ITEMS][PIECES];
#pragma unroll
  for (unsigned u = 0; u < ITEMS; ++u) {
    const unsigned i = u * kThreads + threadIdx.x, row = r0 + i / NB, c = c0 + i % NB * B;
    const T* src = x + (size_t)row * ldx + c;
#pragma unroll
    for (unsigned q = 0; q < PIECES; ++q) {
      raw[u][q] = make_uint4(0, 0, 0, 0);
      if (row < rows && c + (q + 1) * V <= cols) {
        raw[u][q] = *reinterpret_cast<const uint4*>(src + q * V);
      } else if (row < rows && c + q * V < cols) {        // the row ends inside this piece
        T e[V];
#pragma unroll
        for (unsigned j = 0; j < V; ++j) e[j] = c + q * V + j < cols ? src[q * V + j] : from_float<T>(0.0f);
        raw[u][q] = *reinterpret_cast<const uint4*>(e);
      }
    }
  }
  const float ti = __fdiv_rn(1.0f, tensor_scale_of<FORMAT, kThreads>(x, rows, cols, ldx, true, amax, maxima, tensor_scale, part));
  const size_t row_bytes = (size_t)((cols + 31) / 32) * 16;
#pragma unroll
  for (unsigned u = 0; u < ITEMS; ++u) {
    const unsigned i = u * kThreads + threadIdx.x, r = i / NB, blk = i % NB, row = r0 + r, c = c0 + blk * B;
    unsigned word[B / 8];
    const unsigned byte = quantise_words<FORMAT, B, T>(reinterpret_cast<const unsigned*>(raw[u]), ti, word);
    staged_scales[blk / 4 * 512 + (r & 31u) * 16 + (r >> 5) * 4 + (blk & 3u)] = row < rows && c < cols ? (uint8_t)byte : 0;
    if (row < rows && c < row_bytes * 2) {
      uint8_t* out = codes + (size_t)row * row_bytes + c / 2;
      if constexpr (B == 16) *reinterpret_cast<uint2*>(out) = make_uint2(word[0], word[1]);
      else *reinterpret_cast<uint4*>(out) = make_uint4(word[0], word[1], word[2], word[3]);
    }
  }
  __syncthreads();
  write_scales<NB>(staged_scales, scales, cols, r0, c0);
}

// Rows of out that start at multiples of 16 bytes.  A thread takes groups of 16 bytes (their codes lie in one word, the
// values in one block), kRows rows of its place; `wide` threads of a CTA lie along a row, the others in rows below, so that
// no index needs a division.
constexpr unsigned kRows = 4;

template <int FORMAT, typename T>
__global__ void __launch_bounds__(kThreads)
fp4_dequantise_kernel(const uint8_t* __restrict__ codes, const uint8_t* __restrict__ scales, const float* __restrict__ tensor_scale,
                      unsigned rows, unsigned cols, T* __restrict__ out, size_t ldo, unsigned groups, unsigned wide, unsigned strips) {
  constexpr unsigned B = FORMAT == SSGD_MXFP4 ? 32 : 16, G = 16 / sizeof(T);
  pdl_launch_dependents();
  pdl_wait();
  const float ts = FORMAT == SSGD_NVFP4 && tensor_scale ? __ldg(tensor_scale) : 1.0f;
  const unsigned strip = blockIdx.x % strips, high = kThreads / wide;                 // strips of wide groups; rows at a time
  const unsigned g = strip * wide + (threadIdx.x & (wide - 1)), row0 = blockIdx.x / strips * (high * kRows) + threadIdx.x / wide;
  if (g >= groups) return;
  const unsigned c = g * G, row_words = (cols + 31) / 32 * 4, tiles_k = ((cols + B - 1) / B + 3) / 4;
  const uint32_t* words = reinterpret_cast<const uint32_t*>(codes) + c / 8;
  unsigned word[kRows], byte[kRows];
#pragma unroll
  for (unsigned u = 0; u < kRows; ++u) {
    const unsigned row = row0 + u * high;
    word[u] = row < rows ? words[(size_t)row * row_words] : 0u;
    byte[u] = row < rows ? scales[fp4_scale_index(row, c / B, tiles_k)] : 0u;
  }
#pragma unroll
  for (unsigned u = 0; u < kRows; ++u) {
    if (row0 + u * high >= rows) break;
    const unsigned bits = word[u] >> (c % 8 * 4);
    const float scale = __fmul_rn(fp4_scale_value<FORMAT>(byte[u]), ts);
    float v[G];
#pragma unroll
    for (unsigned j = 0; j < G; j += 2) {
      const float2 two = fp4_pair_value(bits >> (4 * j));
      v[j] = __fmul_rn(two.x, scale);
      v[j + 1] = __fmul_rn(two.y, scale);
    }
    T* o = out + (size_t)(row0 + u * high) * ldo + c;
    if (c + G <= cols) {
      if constexpr (sizeof(T) == 4) store4(o, make_float4(v[0], v[1], v[2], v[3]));
      else __stcs(reinterpret_cast<uint4*>(o), make_uint4(pack2(T(), v[0], v[1]), pack2(T(), v[2], v[3]), pack2(T(), v[4], v[5]), pack2(T(), v[6], v[7])));
    } else {
#pragma unroll
      for (unsigned j = 0; j < G; ++j)
        if (c + j < cols) o[j] = from_float<T>(v[j]);
    }
  }
}

// Rows of out that start anywhere.  A warp takes 256 columns of a row: a word of codes to a lane, the block scales to the first
// lanes, then 32 neighbouring values at a time, one to a lane, codes and scale from the lanes that hold them.
template <int FORMAT, typename T>
__global__ void __launch_bounds__(kThreads)
fp4_dequantise_rows_kernel(const uint8_t* __restrict__ codes, const uint8_t* __restrict__ scales, const float* __restrict__ tensor_scale,
                           unsigned rows, unsigned cols, T* __restrict__ out, size_t ldo, unsigned strips) {
  constexpr unsigned B = FORMAT == SSGD_MXFP4 ? 32 : 16, NB = 256 / B;
  pdl_launch_dependents();
  pdl_wait();
  const float ts = FORMAT == SSGD_NVFP4 && tensor_scale ? __ldg(tensor_scale) : 1.0f;
  const unsigned lane = threadIdx.x & 31u, row = blockIdx.x / strips * (kThreads / 32) + (threadIdx.x >> 5), c0 = blockIdx.x % strips * 256;
  if (row >= rows) return;
  const unsigned row_words = (cols + 31) / 32 * 4, blocks = (cols + B - 1) / B, tiles_k = (blocks + 3) / 4;
  const unsigned at = c0 / 8 + lane, block = c0 / B + lane;
  const unsigned word = at < row_words ? reinterpret_cast<const uint32_t*>(codes)[(size_t)row * row_words + at] : 0u;
  const unsigned byte = lane < NB && block < blocks ? scales[fp4_scale_index(row, block, tiles_k)] : 0u;
  const float scale = __fmul_rn(fp4_scale_value<FORMAT>(byte), ts);
  T* o = out + (size_t)row * ldo + c0 + lane;
#pragma unroll
  for (unsigned i = 0; i < 8; ++i) {
    const unsigned code = __shfl_sync(0xFFFFFFFFu, word, 4 * i + lane / 8) >> (lane % 8 * 4);
    const float s = __shfl_sync(0xFFFFFFFFu, scale, (32 * i + lane) / B);
    if (c0 + 32 * i + lane < cols) o[32 * i] = from_float<T>(__fmul_rn(fp4_pair_value(code & 15u).x, s));
  }
}

template <typename T>
bool rows_aligned(const T* x, size_t ldx) { return aligned16(x) && ldx * sizeof(T) % 16 == 0; }

template <int FORMAT, bool ROWS, bool COLS, unsigned THREADS, typename T>
ssgd_status launch_tiles(const T* x, size_t rows, size_t cols, size_t ldx, const float* amax, unsigned maxima, float* tensor_scale,
                            uint8_t* codes, uint8_t* scales, uint8_t* codes_t, uint8_t* scales_t, cudaStream_t s) {
  const size_t tiles_c = (cols + kSide - 1) / kSide, tiles = (rows + kSide - 1) / kSide * tiles_c;
  if (tiles > kMaxGrid) return SSGD_ERR_SIZE;
  const bool words = (reinterpret_cast<uintptr_t>(x) | ldx * sizeof(T)) % 4 == 0;
  const unsigned piece = rows_aligned(x, ldx) ? 16 : words ? 4 : 0;
  auto kernel = fp4_quantise_kernel<FORMAT, ROWS, COLS, THREADS, T>;
  static unsigned long long seen = 0;
  if (!allow_smem(reinterpret_cast<const void*>(kernel), kTileSmem<T>, &seen)) return SSGD_ERR_CUDA;
  launch_kernel(kernel, dim3((unsigned)tiles), dim3(THREADS), kTileSmem<T>, s, true, x, (unsigned)rows, (unsigned)cols, ldx, piece, amax,
                maxima, tensor_scale, codes, scales, codes_t, scales_t, (unsigned)tiles_c);
  return launch_status();
}

// 512 threads for fp32, whose tiles leave room for two CTAs of an SM, and for few 16-bit tiles, where a CTA's own time counts;
// else 256, of which four fit (B200, bf16 both ways: 2048 x 1024 mx 3.2 us with 512, 4.0 with 256; 1999 x 4103 nv 15.1 and 13.8;
// 8192 x 8192 mx 83 and 41).  Registers as the compiler likes them: held to four or five CTAs, 256 threads take 44 and 55 us there.
template <int FORMAT, bool ROWS, bool COLS, typename T>
ssgd_status launch_quantise(const T* x, size_t rows, size_t cols, size_t ldx, const float* amax, unsigned maxima, float* tensor_scale,
                            uint8_t* codes, uint8_t* scales, uint8_t* codes_t, uint8_t* scales_t, cudaStream_t s) {
  DeviceInfo info;
  if (!device_info(&info)) return SSGD_ERR_CUDA;
  if constexpr (ROWS && !COLS && sizeof(T) == 2) {
    const size_t tiles_c = (cols + kSide - 1) / kSide, tiles = (rows + kSide - 1) / kSide * tiles_c;
    if (rows_aligned(x, ldx)) {
      if (tiles > kMaxGrid) return SSGD_ERR_SIZE;
      launch_kernel(fp4_quantise_rows_kernel<FORMAT, T>, dim3((unsigned)tiles), dim3(kThreads), 0, s, true, x, (unsigned)rows, (unsigned)cols, ldx, amax,
                    maxima, tensor_scale, codes, scales, (unsigned)tiles_c);
      return launch_status();
    }
  }
  if (sizeof(T) == 4 || (rows + kSide - 1) / kSide * ((cols + kSide - 1) / kSide) <= (size_t)info.sms * 2)
    return launch_tiles<FORMAT, ROWS, COLS, 512>(x, rows, cols, ldx, amax, maxima, tensor_scale, codes, scales, codes_t, scales_t, s);
  return launch_tiles<FORMAT, ROWS, COLS, sizeof(T) == 4 ? 512 : 256>(x, rows, cols, ldx, amax, maxima, tensor_scale, codes, scales, codes_t, scales_t, s);
}

template <int FORMAT, typename T>
ssgd_status quantise_typed(const T* x, size_t rows, size_t cols, size_t ldx, const float* amax, float* tensor_scale, uint8_t* codes,
                           uint8_t* scales, uint8_t* codes_t, uint8_t* scales_t, cudaStream_t s) {
  unsigned maxima = 0;
  if (FORMAT == SSGD_NVFP4 && !amax && rows * cols > kFusedAmax) {
    DeviceInfo info;
    if (!device_info(&info)) return SSGD_ERR_CUDA;
    const size_t V = 16 / sizeof(T);
    unsigned wide = 32;
    while (wide < kAmaxThreads && wide * V < cols) wide *= 2;
    const size_t strips = (cols + wide * V - 1) / (wide * V), high = kAmaxThreads / wide, most = (size_t)info.sms * kAmaxCtas;
    const unsigned deep = (rows + high * 8 - 1) / (high * 8) * strips < most ? 2 : 8;      // rows of a thread: two where eight leave SMs without work
    const size_t units = (rows + high * deep - 1) / (high * deep) * strips, slots = SSGD_FP4_SCALE_FLOATS - 2;
    const size_t ctas = units < most ? units : most;
    maxima = (unsigned)(ctas < slots ? ctas : slots);
    launch_kernel(deep == 2 ? fp4_amax_kernel<2, T> : fp4_amax_kernel<8, T>, dim3(maxima), dim3(kAmaxThreads), 0, s, true, x, (unsigned)rows,
                  (unsigned)cols, ldx, rows_aligned(x, ldx), wide, (unsigned)strips, (unsigned long long)units, reinterpret_cast<unsigned*>(tensor_scale + 2));
  }
  if (codes && codes_t)
    return launch_quantise<FORMAT, true, true>(x, rows, cols, ldx, amax, maxima, tensor_scale, codes, scales, codes_t, scales_t, s);
  if (codes) return launch_quantise<FORMAT, true, false>(x, rows, cols, ldx, amax, maxima, tensor_scale, codes, scales, codes_t, scales_t, s);
  return launch_quantise<FORMAT, false, true>(x, rows, cols, ldx, amax, maxima, tensor_scale, codes, scales, codes_t, scales_t, s);
}

template <typename T>
ssgd_status quantise_format(const T* x, size_t rows, size_t cols, size_t ldx, int format, const float* amax, float* tensor_scale, uint8_t* codes,
                            uint8_t* scales, uint8_t* codes_t, uint8_t* scales_t, cudaStream_t s) {
  return format == SSGD_MXFP4 ? quantise_typed<SSGD_MXFP4>(x, rows, cols, ldx, amax, tensor_scale, codes, scales, codes_t, scales_t, s)
                              : quantise_typed<SSGD_NVFP4>(x, rows, cols, ldx, amax, tensor_scale, codes, scales, codes_t, scales_t, s);
}

template <int FORMAT, typename T>
ssgd_status launch_dequantise(const uint8_t* codes, const uint8_t* scales, const float* ts, size_t rows, size_t cols, T* out, size_t ldo, cudaStream_t s) {
  if (!rows_aligned(out, rows > 1 ? ldo : 16 / sizeof(T))) {
    const size_t strips = (cols + 255) / 256, high = kThreads / 32, ctas = (rows + high - 1) / high * strips;
    if (ctas > kMaxGrid) return SSGD_ERR_SIZE;
    launch_kernel(fp4_dequantise_rows_kernel<FORMAT, T>, dim3((unsigned)ctas), dim3(kThreads), 0, s, true, codes, scales, ts, (unsigned)rows,
                  (unsigned)cols, out, ldo, (unsigned)strips);
    return launch_status();
  }
  const size_t G = 16 / sizeof(T), groups = (cols + G - 1) / G;
  unsigned wide = 32;
  while (wide < (unsigned)kThreads && wide < groups) wide *= 2;
  const size_t strips = (groups + wide - 1) / wide, high = kThreads / wide * kRows, ctas = (rows + high - 1) / high * strips;
  if (ctas > kMaxGrid) return SSGD_ERR_SIZE;
  launch_kernel(fp4_dequantise_kernel<FORMAT, T>, dim3((unsigned)ctas), dim3(kThreads), 0, s, true, codes, scales, ts, (unsigned)rows, (unsigned)cols, out,
                ldo, (unsigned)groups, wide, (unsigned)strips);
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

ssgd_status ssgd_fp4_quantise_block(const uint64_t* a) {
  if (!a) return SSGD_ERR_NULL;
  return ssgd_fp4_quantise(block_ptr<const void>(a[0]), (int)a[1], a[2], a[3], a[4], (int)a[5], block_ptr<const float>(a[6]), block_ptr<float>(a[7]),
                           block_ptr<uint8_t>(a[8]), block_ptr<uint8_t>(a[9]), block_ptr<uint8_t>(a[10]), block_ptr<uint8_t>(a[11]), block_ptr<void>(a[12]));
}

ssgd_status ssgd_fp4_dequantise_block(const uint64_t* a) {
  if (!a) return SSGD_ERR_NULL;
  return ssgd_fp4_dequantise(block_ptr<const uint8_t>(a[0]), block_ptr<const uint8_t>(a[1]), block_ptr<const float>(a[2]), (int)a[3], a[4], a[5],
                             block_ptr<void>(a[6]), (int)a[7], a[8], block_ptr<void>(a[9]));
}

}  // extern "C"
