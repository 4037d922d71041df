// Cross entropy of a linear head over a large vocabulary, z = h w^T, without the logits: they live in tensor memory only, as
// tiles.  See include/signsgd.h for the contract.
//
//   forward   a product of h and w whose epilogue keeps, for each token and each half tile of the vocabulary, the largest logit and
//             the sum of exponentials below it, and the target's logit; a second kernel joins them (fixed order) to
//             log sum exp and the loss
//   backward  by pieces of the vocabulary: the logits' tiles once more, this time to dz = g (exp(z - lse) - [v = y]), rounded
//             to the operands' type, which is what the two products take that follow: dh += dz w, dw = dz^T h (no operand
//             is transposed in memory, the products read them either way)
// Statistics, losses and all sums are fp32, sums in parts (kSumStages, kGradientStages); dz is the one rounding to 16 bits, as large as that of the
// gradients themselves.  It is divided by its largest entry, a target's g (1 - p), and the products' sums are multiplied by it: where tokens have
// the same g (a mean, a sum) and little idea of their targets, those entries are -1 or close to it and lose little or nothing, where
// -g would be off by the same part of itself for all tokens, up to 2^-8.  In fp16 times 2^14 besides, to keep small probabilities.

#include "half_product.cuh"

namespace {

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kInf = __builtin_inff();

__device__ __forceinline__ float exp2_fast(float x) {   // 2 ulp; exp2(-inf) = 0
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
// A maximum that may be subtracted: -inf - -inf would be NaN where all is -inf so far.
__device__ __forceinline__ float base_of(float top) { return top == -kInf ? 0.0f : top; }

// ---------------------------------------------------------------------------------------------------------------------
// Forward.

// Each thread has one token and half of the tile's columns: a running maximum and sum, nothing to exchange.
struct StatsEpilogue {
  struct Args {
    const int64_t* targets;
    float2* partial;            // [2 * tiles_q][tokens]: maximum, sum
    float* picked;              // [tokens]: the target's logit
    unsigned tokens;
  };
  static constexpr unsigned kBox = 0;
  Box box;
  float top, sum;
  int64_t target;
  unsigned row, part;
  __device__ __forceinline__ StatsEpilogue(const Args&, const Box& b) : box(b) {}
  static __device__ __forceinline__ void prefetch(const Args&) {}
  __device__ __forceinline__ void ahead(const Args&, unsigned) {}
  __device__ __forceinline__ void begin(const Args& a, const HalfPlace& at, unsigned row0, unsigned odd) {
    row = row0 + box.lane;
    part = 2 * at.tile_q + odd;
    top = -kInf;
    sum = 0.0f;
    target = row < a.tokens ? a.targets[row] : -1;
  }
  __device__ __forceinline__ void unit(const Args& a, unsigned column, unsigned left, float (&v)[32]) {
    float(&z)[32] = v;
    if (left < 32) {
#pragma unroll
      for (unsigned q = 0; q < 32; ++q)
        z[q] = q >= left ? -kInf : z[q];
    }
    float m = top;
#pragma unroll
    for (unsigned q = 0; q < 32; ++q) m = fmaxf(m, z[q]);
    const float b = base_of(m);
    float s0 = sum * exp2_fast((top - b) * kLog2e), s1 = 0.0f, s2 = 0.0f, s3 = 0.0f;
#pragma unroll
    for (unsigned q = 0; q < 32; q += 4) {
      s0 += exp2_fast((z[q] - b) * kLog2e);
      s1 += exp2_fast((z[q + 1] - b) * kLog2e);
      s2 += exp2_fast((z[q + 2] - b) * kLog2e);
      s3 += exp2_fast((z[q + 3] - b) * kLog2e);
    }
    sum = (s0 + s1) + (s2 + s3);
    top = m;
    const int64_t at = target - (int64_t)column;
    if (at >= 0 && at < (int64_t)left) {
      float picked = 0.0f;
      unsigned which = (unsigned)at;
#pragma unroll
      for (unsigned q = 0; q < 32; ++q) {
        asm volatile("" : "+r"(which));           // or the compiler makes an index of it, and puts the sums into local memory
        picked = which == q ? z[q] : picked;
      }
      a.picked[row] = picked;
    }
  }
  __device__ __forceinline__ void end(const Args& a, const HalfPlace&, unsigned) {
    if (row < a.tokens) a.partial[(size_t)part * a.tokens + row] = make_float2(top, sum);
  }
  __device__ __forceinline__ void finish(const Args&) {}
};

// What the backward pass has to know of a token.
constexpr uint8_t kCounts = 0, kIgnored = 1, kIgnoredNotFinite = 2;

// Two parts of a sum of exponentials, each beside its maximum.
__device__ __forceinline__ float2 join(float2 a, float2 b) {
  const float m = fmaxf(a.x, b.x), base = base_of(m);
  return make_float2(m, a.y * exp2_fast((a.x - base) * kLog2e) + b.y * exp2_fast((b.x - base) * kLog2e));
}

// A few tokens: the weight's bytes are all that counts, and a warp takes four rows of it at a time against tokens that lie in shared memory,
// in fp32.  (Whole forward passes on B200, weights from HBM, this kernel / tiles of tensor-core products: 30522 x 1024 with one token 16.5 /
// 19.0 us, two 18.3 / 19.1, four 24.9 / 19.8; 131072 x 4096 165 / 197, 176 / 196, 222 / 191; so up to two: more registers and conversions
// per byte from there on.  With the 62 MB of 30522 x 1024 in L2 12.5, 15.1, 20.9 / 22.7.)
constexpr unsigned kFewRows = 4, kFewWarps = 8;
constexpr size_t kFewSmem = 98304;

template <unsigned TOKENS, typename T>
__global__ void __launch_bounds__(32 * kFewWarps, 2)
xent_few_kernel(const T* __restrict__ h, size_t ldh, const T* __restrict__ w, size_t ldw, unsigned tokens, unsigned vocab, unsigned width,
                const int64_t* __restrict__ targets, float2* __restrict__ partial, float* __restrict__ picked) {
  // [token][half of eight][piece of 128][lane's four]: lanes read 16 bytes side by side
  extern __shared__ float few_smem[];
  __shared__ float2 parts[kFewWarps][kFewRows * TOKENS];
  pdl_launch_dependents();
  pdl_wait();
  const unsigned warp = threadIdx.x >> 5, lane = threadIdx.x & 31u, pieces = (width + 255) / 256;
  for (unsigned i = threadIdx.x; i < TOKENS * pieces * 256; i += 32 * kFewWarps) {
    const unsigned t = i / (pieces * 256), c = i % (pieces * 256);
    few_smem[((t * 2 + (c >> 2 & 1u)) * pieces + (c >> 8)) * 128 + (c >> 3 & 31u) * 4 + (c & 3u)] = t < tokens && c < width ? to_float(h[(size_t)t * ldh + c]) : 0.0f;
  }
  __syncthreads();

  // lane r * TOKENS + t keeps the running maximum and sum of the rows r of token t
  const unsigned my_row = lane / TOKENS, my_token = lane % TOKENS;
  const bool keeps = lane < kFewRows * TOKENS && my_token < tokens;
  const int64_t target = keeps ? targets[my_token] : -1;
  float top = -kInf, sum = 0.0f;
  for (unsigned row0 = (blockIdx.x * kFewWarps + warp) * kFewRows; row0 < vocab; row0 += gridDim.x * kFewWarps * kFewRows) {
    float z[kFewRows][TOKENS];
#pragma unroll
    for (unsigned r = 0; r < kFewRows; ++r)
#pragma unroll
      for (unsigned t = 0; t < TOKENS; ++t) z[r][t] = 0.0f;
#pragma unroll 2
    for (unsigned p = 0; p < pieces; ++p) {
      const unsigned c = p * 256 + lane * 8;
      uint4 q[kFewRows];
#pragma unroll
      for (unsigned r = 0; r < kFewRows; ++r)
        q[r] = c < width && row0 + r < vocab ? __ldg(reinterpret_cast<const uint4*>(w + (size_t)(row0 + r) * ldw + c)) : make_uint4(0, 0, 0, 0);
      if (c < width && c + 8 > width) {           // what lies behind the last column may be anything
        const unsigned left = width - c;
#pragma unroll
        for (unsigned r = 0; r < kFewRows; ++r) {
          unsigned* words = &q[r].x;
#pragma unroll
          for (unsigned k = 0; k < 4; ++k) words[k] = 2 * k + 1 < left ? words[k] : 2 * k < left ? words[k] & 0xFFFFu : 0u;
        }
      }
#pragma unroll
      for (unsigned t = 0; t < TOKENS; ++t) {
        const float4 a = *reinterpret_cast<const float4*>(few_smem + ((t * 2) * pieces + p) * 128 + lane * 4);
        const float4 b = *reinterpret_cast<const float4*>(few_smem + ((t * 2 + 1) * pieces + p) * 128 + lane * 4);
#pragma unroll
        for (unsigned r = 0; r < kFewRows; ++r) {
          float s = z[r][t];
          s = fmaf(low_to_float(T(), q[r].x), a.x, s);
          s = fmaf(high_to_float(T(), q[r].x), a.y, s);
          s = fmaf(low_to_float(T(), q[r].y), a.z, s);
          s = fmaf(high_to_float(T(), q[r].y), a.w, s);
          s = fmaf(low_to_float(T(), q[r].z), b.x, s);
          s = fmaf(high_to_float(T(), q[r].z), b.y, s);
          s = fmaf(low_to_float(T(), q[r].w), b.z, s);
          z[r][t] = fmaf(high_to_float(T(), q[r].w), b.w, s);
        }
      }
    }
    float mine = 0.0f;
#pragma unroll
    for (unsigned r = 0; r < kFewRows; ++r)
#pragma unroll
      for (unsigned t = 0; t < TOKENS; ++t) {
        float s = z[r][t];
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xFFFFFFFFu, s, o);
        mine = lane == r * TOKENS + t ? s : mine;
      }
    if (keeps && row0 + my_row < vocab) {
      if (target == (int64_t)(row0 + my_row)) picked[my_token] = mine;
      const float2 both = join(make_float2(top, sum), make_float2(mine, 1.0f));
      top = both.x;
      sum = both.y;
    }
  }
  if (lane < kFewRows * TOKENS) parts[warp][lane] = make_float2(top, sum);
  __syncthreads();
  if (threadIdx.x < TOKENS && threadIdx.x < tokens) {
    float2 all = make_float2(-kInf, 0.0f);
    for (unsigned k = 0; k < kFewWarps; ++k)
#pragma unroll
      for (unsigned r = 0; r < kFewRows; ++r) all = join(all, parts[k][r * TOKENS + threadIdx.x]);
    partial[(size_t)blockIdx.x * tokens + threadIdx.x] = all;
  }
}

// Joins the parts of TOKENS tokens a CTA (1 or 8), its other threads side by side along the parts; then the losses, and a look at the
// ignored tokens' rows of h: one that is not finite must not reach dw through 0 * inf.
template <unsigned TOKENS, typename T>
__global__ void __launch_bounds__(256)
xent_join_kernel(const float2* __restrict__ partial, const float* __restrict__ picked, const int64_t* __restrict__ targets, int64_t ignore, unsigned tokens,
                 unsigned parts, unsigned vocab, const T* __restrict__ h, size_t ldh, unsigned width, float* __restrict__ losses, float* __restrict__ lse,
                 uint8_t* __restrict__ kinds) {
  constexpr unsigned kSlices = 256 / TOKENS;
  __shared__ float2 part[TOKENS == 1 ? 8 : kSlices][TOKENS];
  pdl_launch_dependents();
  pdl_wait();
  const unsigned i = threadIdx.x % TOKENS, slice = threadIdx.x / TOKENS, t0 = blockIdx.x * TOKENS, t = t0 + i;
  const bool mine = threadIdx.x < TOKENS && t < tokens;
  const int64_t y = mine ? targets[t] : 0;
  float2 sum = make_float2(-kInf, 0.0f);
  if (t < tokens) {
    for (unsigned p0 = slice; p0 < parts; p0 += 8 * kSlices) {
      float2 v[8];
#pragma unroll
      for (unsigned u = 0; u < 8; ++u) v[u] = p0 + u * kSlices < parts ? partial[(size_t)(p0 + u * kSlices) * tokens + t] : make_float2(-kInf, 0.0f);
      float m = sum.x;
#pragma unroll
      for (unsigned u = 0; u < 8; ++u) m = fmaxf(m, v[u].x);
      const float b = base_of(m);
      sum.y *= exp2_fast((sum.x - b) * kLog2e);
#pragma unroll
      for (unsigned u = 0; u < 8; ++u) sum.y += v[u].y * exp2_fast((v[u].x - b) * kLog2e);
      sum.x = m;
    }
  }
  if (TOKENS == 1) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) sum = join(sum, make_float2(__shfl_xor_sync(0xFFFFFFFFu, sum.x, o), __shfl_xor_sync(0xFFFFFFFFu, sum.y, o)));
    if (threadIdx.x % 32 == 0) part[threadIdx.x / 32][0] = sum;
  } else {
    part[slice][i] = sum;
  }
  __syncthreads();
  if (mine) {
    sum = part[0][i];
#pragma unroll
    for (unsigned k = 1; k < (TOKENS == 1 ? 8 : kSlices); ++k) sum = join(sum, part[k][i]);
    const bool ignored = y == ignore, inside = y >= 0 && y < (int64_t)vocab;
    // a target that is neither ignored nor in the vocabulary: NaN, here and in the gradients
    const float log_sum = logf(sum.y), l = inside || ignored ? sum.x + log_sum : __uint_as_float(0x7FC00000u);
    const float loss = ignored ? 0.0f : inside ? (sum.x - picked[t]) + log_sum : l;
    losses[t] = loss;
    lse[t] = l;
    lse[tokens + t] = loss;
    if (!ignored) kinds[t] = kCounts;
  }
  // a warp for each ignored token
  for (unsigned k = threadIdx.x / 32; k < TOKENS; k += 8) {
    const unsigned row = t0 + k;
    if (row >= tokens || targets[row] != ignore) continue;
    bool finite = true;
#pragma unroll 8
    for (unsigned c = threadIdx.x % 32; c < width; c += 32) finite &= isfinite(to_float(h[(size_t)row * ldh + c])) != 0;
    finite = __all_sync(0xFFFFFFFFu, finite);
    if (threadIdx.x % 32 == 0) kinds[row] = finite ? kIgnored : kIgnoredNotFinite;
  }
}

// ---------------------------------------------------------------------------------------------------------------------
// Backward.

// Before the products: the scale of dz, and, only where an ignored token's row of h is not finite, a copy of h with the
// ignored rows zero, which dw's product then takes for h.
struct Prepared {
  unsigned copied;              // h's copy is to be taken
  float scale, unscale;         // of dz
  unsigned unused;
};
template <typename T>
__global__ void __launch_bounds__(256)
xent_prepare_kernel(const uint8_t* __restrict__ kinds, const float* __restrict__ lse, const float* __restrict__ g, size_t g_stride, unsigned tokens,
                    const T* __restrict__ h, size_t ldh, unsigned width, T* __restrict__ copy, size_t ldc, Prepared* __restrict__ out) {
  __shared__ unsigned part[8];
  pdl_launch_dependents();
  pdl_wait();
  unsigned bad = 0;
#pragma unroll 8
  for (unsigned t = threadIdx.x; t < tokens; t += 256) bad |= kinds[t] == kIgnoredNotFinite;
  bad = __syncthreads_or((int)bad) != 0;
  if (blockIdx.x == 0) {
    unsigned top = 0;                                       // a magnitude's bits are ordered as it is
    for (unsigned t0 = threadIdx.x; t0 < tokens; t0 += 8 * 256) {      // eight in flight: one CTA, and the products wait for it
      float loss[8], of[8];
      bool counts[8];
#pragma unroll
      for (unsigned u = 0; u < 8; ++u) {
        const unsigned t = t0 + u * 256;
        counts[u] = t < tokens && kinds[t] == kCounts;
        loss[u] = t < tokens ? lse[tokens + t] : 0.0f;
        of[u] = t < tokens ? g[t * g_stride] : 0.0f;
      }
#pragma unroll
      for (unsigned u = 0; u < 8; ++u) {                    // probabilities below 2^-24 may be missing from a sum of 1; a loss or g that is not finite leaves the others' factor alone
        const unsigned entry = __float_as_uint(of[u] * fmaxf(-expm1f(-loss[u]), 2.4e-7f)) & 0x7FFFFFFFu;
        if (counts[u] && entry < 0x7F800000u) top = max(top, entry);
      }
    }
    top = __reduce_max_sync(0xFFFFFFFFu, top);
    if (threadIdx.x % 32 == 0) part[threadIdx.x / 32] = top;
    __syncthreads();
    for (unsigned k = 0; k < 8; ++k) top = max(top, part[k]);
    if (threadIdx.x == 0) {
      constexpr float kTop = std::is_same<T, __half>::value ? 16384.0f : 1.0f;
      const float most = __uint_as_float(top);
      Prepared p = {bad, 1.0f, 1.0f, 0};
      if (most >= 7.9e-31f && most <= 1.3e36f) {            // 2^-100 .. 2^120: both factors are fp32 numbers
        p.scale = __fdiv_rn(kTop, most);
        p.unscale = most * (1.0f / kTop);
      } else if (top > 0) {                                 // out there by a power of two that leaves at most 2^14, which fp16 holds
        const int e = most < 1.0f ? 114 : -114;
        p.scale = __uint_as_float((unsigned)(127 + e) << 23);
        p.unscale = __uint_as_float((unsigned)(127 - e) << 23);
      }
      *out = p;
    }
  }
  if (!bad) return;
  for (unsigned t = blockIdx.x; t < tokens; t += gridDim.x) {
    const bool keep = kinds[t] == kCounts;
    for (unsigned c = threadIdx.x; c < width; c += 256) copy[(size_t)t * ldc + c] = keep ? h[(size_t)t * ldh + c] : from_float<T>(0.0f);
  }
}

template <typename T>
struct GradEpilogue {
  struct Args {
    CUtensorMap dz;             // [tokens][columns of this piece]
    const int64_t* targets;
    const float* lse;           // [2][tokens], see the join
    const float* g;
    const uint8_t* kinds;
    const Prepared* prepared;
    size_t g_stride;
    unsigned tokens, first;     // first: column of the vocabulary at which the piece begins
  };
  static constexpr unsigned kBox = 4096;      // two boxes in turn
  Box box;
  float lse, g, miss;           // miss: the target's probability less one
  int64_t target;
  unsigned row0, half;
  bool counts;
  __device__ __forceinline__ GradEpilogue(const Args&, const Box& b) : box(b), half(0) {}
  static __device__ __forceinline__ void prefetch(const Args& a) { prefetch_tensor_map(&a.dz); }
  __device__ __forceinline__ void ahead(const Args&, unsigned) {}
  __device__ __forceinline__ void begin(const Args& a, const HalfPlace&, unsigned first_row, unsigned) {
    row0 = first_row;
    const unsigned row = row0 + box.lane;
    counts = false;
    if (row >= a.tokens) return;
    counts = a.kinds[row] == kCounts;
    lse = a.lse[row];
    // from the loss, -log p: a difference of probabilities would keep nothing of a token that is sure of its target
    miss = expm1f(-a.lse[a.tokens + row]);
    g = a.g[row * a.g_stride] * a.prepared->scale;
    target = a.targets[row] - (int64_t)a.first;
  }
  __device__ __forceinline__ void unit(const Args& a, unsigned column, unsigned, float (&v)[32]) {
    if (counts) {
#pragma unroll
      for (unsigned q = 0; q < 32; ++q) v[q] = exp2_fast((v[q] - lse) * kLog2e);
      const int64_t at = target - (int64_t)column;
      if (at >= 0 && at < 32) {
#pragma unroll
        for (unsigned q = 0; q < 32; ++q) v[q] = (unsigned)at == q ? miss : v[q];
      }
#pragma unroll
      for (unsigned q = 0; q < 32; ++q) v[q] *= g;
    } else {
#pragma unroll
      for (unsigned q = 0; q < 32; ++q) v[q] = 0.0f;
    }
    half ^= 2048;
    box.sent_but_last();
    box.template put16<T>(half, v);
    box.fence();
    box.send(a.dz, half, column, row0, 0);
  }
  __device__ __forceinline__ void end(const Args&, const HalfPlace&, unsigned) {}
  __device__ __forceinline__ void finish(const Args&) { box.finish(); }
};

// dh: rows of tokens, those that are ignored zero.  Where the vocabulary is in several pieces the sums so far are in fp32; where k
// is split, each split has a plane of its own.
template <typename T>
struct TokensEpilogue {
  struct Args {
    const uint8_t* kinds;
    const Prepared* prepared;
    float* sums;                // [splits][tokens][width], or null
    T* out;                     // null while pieces are to come, and where splits are joined later
    size_t ldo;
    unsigned tokens, width, add;
  };
  static constexpr unsigned kBox = 4096;
  Box box;
  float unscale;
  unsigned row0, split;
  bool counts;
  __device__ __forceinline__ TokensEpilogue(const Args& a, const Box& b) : box(b) { unscale = a.prepared->unscale; }
  static __device__ __forceinline__ void prefetch(const Args&) {}
  __device__ __forceinline__ void ahead(const Args&, unsigned) {}
  __device__ __forceinline__ void begin(const Args& a, const HalfPlace& at, unsigned first_row, unsigned) {
    row0 = first_row;
    split = at.split;
    counts = row0 + box.lane < a.tokens && a.kinds[row0 + box.lane] == kCounts;
  }
  __device__ __forceinline__ void unit(const Args& a, unsigned column, unsigned left, float (&v)[32]) {
    const float by = a.out ? unscale : 1.0f;
    if (!a.add) {
#pragma unroll
      for (unsigned q = 0; q < 32; ++q) v[q] = counts ? v[q] * by : 0.0f;
    } else {
#pragma unroll
      for (unsigned q = 0; q < 32; ++q) v[q] = counts ? v[q] : 0.0f;
    }
    const unsigned rows = min(32u, a.tokens - row0);
    float* sums = a.sums + ((size_t)split * a.tokens + row0) * a.width + column;
    T* out = a.out + (size_t)row0 * a.ldo + column;
    if (a.add && a.out) box.rows_join(sums, a.width, out, a.ldo, rows, left, v, [by](float old, float now) { return (old + now) * by; });
    else if (a.add) box.rows_join(sums, a.width, sums, a.width, rows, left, v, [](float old, float now) { return old + now; });
    else if (a.out) box.rows_out(out, a.ldo, rows, left, v);
    else box.rows_out(sums, a.width, rows, left, v);
  }
  __device__ __forceinline__ void end(const Args&, const HalfPlace&, unsigned) {}
  __device__ __forceinline__ void finish(const Args&) {}
};

// The planes' sums, in order; a thread's four elements a CTA's width apart, eight loads in flight.
template <typename T>
__global__ void __launch_bounds__(256)
xent_planes_kernel(const float* __restrict__ sums, unsigned planes, size_t plane, const Prepared* __restrict__ prepared, unsigned width, T* __restrict__ out,
                   size_t ldo) {
  pdl_launch_dependents();
  pdl_wait();
  const size_t i0 = (size_t)blockIdx.x * 1024 + threadIdx.x;
  float s[4] = {0.0f, 0.0f, 0.0f, 0.0f};
  for (unsigned p = 0; p < planes; p += 2) {
    float v[2][4];
#pragma unroll
    for (unsigned u = 0; u < 2; ++u)
#pragma unroll
      for (unsigned k = 0; k < 4; ++k) v[u][k] = p + u < planes && i0 + 256 * k < plane ? __ldcs(sums + (p + u) * plane + i0 + 256 * k) : 0.0f;
#pragma unroll
    for (unsigned u = 0; u < 2; ++u)
#pragma unroll
      for (unsigned k = 0; k < 4; ++k) s[k] += v[u][k];
  }
  const float unscale = prepared->unscale;
#pragma unroll
  for (unsigned k = 0; k < 4; ++k) {
    const size_t i = i0 + 256 * k;
    if (i < plane) out[i / width * ldo + i % width] = from_float<T>(s[k] * unscale);
  }
}

// dw: rows of the vocabulary.
template <typename T>
struct WeightEpilogue {
  struct Args {
    const Prepared* prepared;
    T* out;
    size_t ldo;
    unsigned rows;
  };
  static constexpr unsigned kBox = 4096;
  Box box;
  float unscale;
  unsigned row0;
  __device__ __forceinline__ WeightEpilogue(const Args& a, const Box& b) : box(b) { unscale = a.prepared->unscale; }
  static __device__ __forceinline__ void prefetch(const Args&) {}
  __device__ __forceinline__ void ahead(const Args&, unsigned) {}
  __device__ __forceinline__ void begin(const Args&, const HalfPlace&, unsigned first_row, unsigned) { row0 = first_row; }
  __device__ __forceinline__ void unit(const Args& a, unsigned column, unsigned left, float (&v)[32]) {
#pragma unroll
    for (unsigned q = 0; q < 32; ++q) v[q] *= unscale;
    box.rows_out(a.out + (size_t)row0 * a.ldo + column, a.ldo, min(32u, a.rows - row0), left, v);
  }
  __device__ __forceinline__ void end(const Args&, const HalfPlace&, unsigned) {}
  __device__ __forceinline__ void finish(const Args&) {}
};

// Rows of 16-bit elements at any place and strides to rows that asynchronous copies can read, of two matrices in one launch: eight elements
// a thread, zeros behind the last column.
struct Scattered {
  const uint16_t* from;
  uint16_t* to;
  size_t ld, step, rows;
};
__global__ void __launch_bounds__(256)
xent_align_kernel(const Scattered a, const Scattered b, unsigned cols, size_t ldo) {
  pdl_launch_dependents();
  pdl_wait();
  const unsigned pieces = (unsigned)(ldo / 8);
  const size_t i = (size_t)blockIdx.x * 256 + threadIdx.x, all = i / pieces;
  const unsigned c = (unsigned)(i - all * pieces) * 8;
  if (all >= a.rows + b.rows) return;
  const bool second = all >= a.rows;
  const Scattered& m = second ? b : a;
  const size_t row = second ? all - a.rows : all;
  const uint16_t* from = m.from + row * m.ld + c * m.step;
  unsigned v[8];
#pragma unroll
  for (unsigned k = 0; k < 8; ++k) v[k] = c + k < cols ? from[k * m.step] : 0u;
  *reinterpret_cast<uint4*>(m.to + row * ldo + c) = make_uint4(v[0] | v[1] << 16, v[2] | v[3] << 16, v[4] | v[5] << 16, v[6] | v[7] << 16);
}

// ---------------------------------------------------------------------------------------------------------------------
// Host side.

constexpr size_t kSide = (size_t)1 << 30;
inline size_t up(size_t n, size_t k) { return (n + k - 1) / k * k; }

// Stages between two times that a logit's sum is taken (each takes the threads 1500 clocks of 256 columns; four: 102 us for 2048 x 30522 x 1024).
// The backward pass makes its logits by the same parts: what they are off beyond the forward pass's, whose log sum exp is taken from them, would be
// a factor of all probabilities (a row of dz for a width of 16384 and logits near 40 sums to 2e-3 with one part, to 3e-6 with these).
constexpr int kSumStages = 8;
// The same for the gradients' products, 2048 of the vocabulary or of the tokens: 2e-5 of a sum whose terms have one sign, a tenth of fp16's
// rounding.  In fp16, one part / these: dh over 131072 words that share a direction off by 2.1e-3 / 2.3e-4, dw of 65536 tokens by 4e-4 /
// 1.2e-5.  Whole training passes with both kinds of parts / without: 8192 x 32768 x 4096 6.9 / 6.7 ms, 2048 x 30522 x 1024 456 / 443 us,
// 777 x 5003 x 1111 105 / 103 us.
constexpr int kGradientStages = 32;
constexpr size_t kFewTokens = 2, kFewCtas = 2;      // see xent_few_kernel; CTAs of an SM

struct HeadSizes {
  size_t parts;                             // partial statistics of a token
  size_t forward_bytes;
  size_t piece, pieces;                     // columns of the vocabulary at a time
  unsigned splits;                          // of dh's k, the vocabulary
  size_t prepared, copy, copy_ld, dz, dz_ld, sums, backward_bytes;       // offsets and row lengths
};

// Pieces: dz of a piece is at most 2^27 numbers (256 MB), in whole 256 columns; 256 columns where more than 2^19 tokens make that more.
constexpr size_t kPieceElements = (size_t)1 << 27;
inline HalfForm stats_form(size_t T, size_t V, size_t D, int sms) {
  HalfProduct p = {};
  p.P = T; p.Q = V; p.K = D; p.batch = 1;
  return half_form(p, 1, 1, sms);
}
inline bool head_sizes(size_t T, size_t V, size_t D, int sms, HeadSizes* s) {
  if (T < 1 || V < 1 || D < 1 || T > kSide || V > kSide || D > kSide || T > ((size_t)1 << 44) / V || T > ((size_t)1 << 44) / D) return false;
  // of a token: two for each tile of the form that the forward product takes, or one for each CTA of the streaming kernel
  s->parts = 2 * ((V + stats_form(T, V, D, sms).nt - 1) / stats_form(T, V, D, sms).nt);
  if (T <= kFewTokens && s->parts < kFewCtas * (size_t)sms) s->parts = kFewCtas * (size_t)sms;
  s->forward_bytes = up(T * 4, 16) + s->parts * T * sizeof(float2);
  const size_t columns = up(V, 256);
  s->piece = up(kPieceElements / T < 256 ? 256 : kPieceElements / T / 256 * 256, 256);
  if (s->piece > columns) s->piece = columns;
  s->pieces = (V + s->piece - 1) / s->piece;
  // dh has few tiles and a long k: split k, where that is faster, by what the products take and the planes of sums take to be added (22
  // bytes of HBM a clock and SM, a launch)
  HalfProduct dh = {};
  dh.P = T; dh.Q = D; dh.K = V; dh.batch = 1;
  s->splits = 1;
  unsigned long long least = 0;
  (void)half_form(dh, 1, 1, sms, &least);
  for (unsigned splits = 2; splits <= 16 && s->pieces == 1 && V >= 256 * (size_t)splits && splits * T * D <= kPieceElements; ++splits) {
    unsigned long long clocks = 0;
    (void)half_form(dh, 1, splits, sms, &clocks);
    clocks += 12000 + 2 * splits * T * D * 4 / (22 * (size_t)sms);
    if (clocks < least) {
      least = clocks;
      s->splits = splits;
    }
  }
  size_t at = 0;
  s->prepared = at; at += 64;
  s->copy = at; s->copy_ld = up(D, 8); at += up(T * s->copy_ld * 2, 128);
  s->dz = at; s->dz_ld = s->piece; at += up(T * s->dz_ld * 2, 128);
  s->sums = at;
  if (s->pieces > 1 || s->splits > 1) at += up(s->splits * T * D * 4, 128);
  s->backward_bytes = at;
  return true;
}

ssgd_status check_head(const void* h, size_t ldh, const void* w, size_t ldw, int dtype, size_t T, size_t V, size_t D, const int64_t* targets, const void* ws,
                       const unsigned* status) {
  if (dtype != SSGD_BF16 && dtype != SSGD_F16) return SSGD_ERR_ARG;
  if (V < 1 || D < 1 || T > kSide || V > kSide || D > kSide || ldh < D || ldw < D || ldh >= (size_t)1 << 38 || ldw >= (size_t)1 << 38) return SSGD_ERR_SIZE;
  if (T == 0) return SSGD_OK;
  if (!h || !w || !targets || !ws || !status) return SSGD_ERR_NULL;
  if (!aligned16(h) || !aligned16(w) || ldh % 8 != 0 || ldw % 8 != 0 || !aligned16(ws) || (reinterpret_cast<uintptr_t>(targets) & 7u) ||
      (reinterpret_cast<uintptr_t>(status) & 3u))
    return SSGD_ERR_ALIGN;
  return SSGD_OK;
}

template <typename T>
ssgd_status head_forward(const T* h, size_t ldh, const T* w, size_t ldw, size_t tokens, size_t vocab, size_t width, const int64_t* targets, int64_t ignore,
                         float* losses, float* lse, uint8_t* kinds, void* ws, unsigned* status, unsigned starve, int sms, cudaStream_t s) {
  float* picked = static_cast<float*>(ws);
  float2* partial = reinterpret_cast<float2*>(static_cast<char*>(ws) + up(tokens * 4, 16));
  unsigned parts;
  const size_t few = tokens < kFewTokens ? 1 : kFewTokens, few_smem = few * ((width + 255) / 256) * 256 * 4;
  if (tokens <= kFewTokens && few_smem <= kFewSmem && starve == 0) {
    const size_t groups = (vocab + kFewWarps * kFewRows - 1) / (kFewWarps * kFewRows), most = kFewCtas * (size_t)sms;
    parts = (unsigned)(groups < most ? groups : most);
    auto kernel = few == 1 ? xent_few_kernel<1, T> : xent_few_kernel<2, T>;
    static unsigned long long seen[2] = {0, 0};
    if (!allow_smem(reinterpret_cast<const void*>(kernel), kFewSmem, &seen[few - 1])) return SSGD_ERR_CUDA;
    launch_kernel(kernel, dim3(parts), dim3(32 * kFewWarps), few_smem, s, true, h, ldh, w, ldw, (unsigned)tokens, (unsigned)vocab, (unsigned)width, targets,
                  partial, picked);
    const ssgd_status st = launch_status();
    if (st != SSGD_OK) return st;
  } else {
    HalfProduct p = {};
    p.p = {h, nullptr, ldh, 0, false};
    p.q = {w, nullptr, ldw, 0, false};
    p.P = tokens; p.Q = vocab; p.K = width; p.batch = 1;
    p.bf16 = std::is_same<T, __nv_bfloat16>::value;
    p.status = status;
    p.starve = starve;
    const HalfForm form = stats_form(tokens, vocab, width, sms);
    const StatsEpilogue::Args args = {targets, partial, picked, (unsigned)tokens};
    const ssgd_status st = launch_half<StatsEpilogue, 1, kSumStages, kBothByK>(p, args, form, 1, sms, s);
    if (st != SSGD_OK) return st;
    parts = 2 * (unsigned)((vocab + form.nt - 1) / form.nt);
  }
  if (tokens <= 512)
    launch_kernel(xent_join_kernel<1, T>, dim3((unsigned)tokens), dim3(256), 0, s, true, partial, picked, targets, ignore, (unsigned)tokens, parts,
                  (unsigned)vocab, h, ldh, (unsigned)width, losses, lse, kinds);
  else
    launch_kernel(xent_join_kernel<8, T>, dim3((unsigned)(tokens + 7) / 8), dim3(256), 0, s, true, partial, picked, targets, ignore, (unsigned)tokens, parts,
                  (unsigned)vocab, h, ldh, (unsigned)width, losses, lse, kinds);
  return launch_status();
}

struct HeadBackward {
  const void *h, *w;
  size_t ldh, ldw, T, V, D;
  const int64_t* targets;
  const float* lse;
  const uint8_t* kinds;
  const float* g;
  size_t g_stride;
  void* dh;
  size_t lddh;
  void* dw;
  int dw_type;
  size_t lddw;
  char* ws;
  unsigned* status;
};

template <typename O>
ssgd_status weight_product(const HalfProduct& p, const HeadBackward& b, const Prepared* prepared, size_t first, size_t rows, int sms, cudaStream_t s) {
  const typename WeightEpilogue<O>::Args args = {prepared, static_cast<O*>(b.dw) + first * b.lddw, b.lddw, (unsigned)rows};
  return launch_half<WeightEpilogue<O>, 1, kGradientStages, kBothByRows>(p, args, half_form(p, 1, 1, sms), 1, sms, s);
}

template <typename T>
ssgd_status head_backward(const HeadBackward& b, int sms, cudaStream_t s) {
  constexpr bool kBf16 = std::is_same<T, __nv_bfloat16>::value;
  HeadSizes z;
  if (!head_sizes(b.T, b.V, b.D, sms, &z)) return SSGD_ERR_SIZE;
  const T *h = static_cast<const T*>(b.h), *w = static_cast<const T*>(b.w);
  Prepared* prepared = reinterpret_cast<Prepared*>(b.ws + z.prepared);
  T *copy = reinterpret_cast<T*>(b.ws + z.copy), *dz = reinterpret_cast<T*>(b.ws + z.dz);
  float* sums = reinterpret_cast<float*>(b.ws + z.sums);
  const unsigned tokens = (unsigned)b.T, width = (unsigned)b.D;
  launch_kernel(xent_prepare_kernel<T>, dim3(tokens < (unsigned)sms * 4 ? tokens : (unsigned)sms * 4), dim3(256), 0, s, true, b.kinds, b.lse, b.g, b.g_stride,
                tokens, h, b.ldh, width, copy, z.copy_ld, prepared);
  ssgd_status st = launch_status();
  for (size_t first = 0; st == SSGD_OK && first < b.V; first += z.piece) {
    const size_t columns = b.V - first < z.piece ? b.V - first : z.piece;
    const T* w_piece = w + first * b.ldw;
    const bool last = first + columns == b.V;
    HalfProduct p = {};
    p.batch = 1;
    p.bf16 = kBf16;
    p.status = b.status;
    p.p = {h, nullptr, b.ldh, 0, false};
    p.q = {w_piece, nullptr, b.ldw, 0, false};
    p.P = b.T; p.Q = columns; p.K = b.D;
    typename GradEpilogue<T>::Args grad = {{}, b.targets, b.lse, b.g, b.kinds, prepared, b.g_stride, tokens, (unsigned)first};
    if (!box_map(&grad.dz, dz, kBf16, b.T, columns, z.dz_ld, 1, 0)) return SSGD_ERR_CUDA;
    st = launch_half<GradEpilogue<T>, 1, kSumStages, kBothByK>(p, grad, half_form(p, 1, 1, sms), 1, sms, s);
    if (st != SSGD_OK) break;
    if (b.dh) {
      p.p = {dz, nullptr, z.dz_ld, 0, false};
      p.q = {w_piece, nullptr, b.ldw, 0, true};
      p.P = b.T; p.Q = b.D; p.K = columns;
      T* out = last && z.splits == 1 ? static_cast<T*>(b.dh) : nullptr;
      const typename TokensEpilogue<T>::Args args = {b.kinds, prepared, z.pieces > 1 || z.splits > 1 ? sums : nullptr, out, b.lddh, tokens, width, first > 0};
      st = launch_half<TokensEpilogue<T>, 1, kGradientStages, kQByRows>(p, args, half_form(p, 1, z.splits, sms), z.splits, sms, s);
      if (st == SSGD_OK && z.splits > 1) {
        const size_t plane = b.T * b.D;
        launch_kernel(xent_planes_kernel<T>, dim3(grid_for((plane + 1023) / 1024)), dim3(256), 0, s, true, sums, z.splits, plane, prepared, width,
                      static_cast<T*>(b.dh), b.lddh);
        st = launch_status();
      }
    }
    if (st == SSGD_OK && b.dw) {
      p.p = {dz, nullptr, z.dz_ld, 0, true};
      p.q = {h, nullptr, b.ldh, 0, true};
      p.P = columns; p.Q = b.D; p.K = b.T;
      HalfProduct other = p;
      other.q_other = copy;
      other.q_choice = &prepared->copied;
      other.q_other_ld = z.copy_ld;
      st = b.dw_type == SSGD_F32    ? weight_product<float>(other, b, prepared, first, columns, sms, s)
           : b.dw_type == SSGD_BF16 ? weight_product<__nv_bfloat16>(other, b, prepared, first, columns, sms, s)
                                    : weight_product<__half>(other, b, prepared, first, columns, sms, s);
    }
  }
  return st;
}

ssgd_status checked_forward(const void* h, size_t ldh, const void* w, size_t ldw, int dtype, size_t T, size_t V, size_t D, const int64_t* targets,
                            int64_t ignore, float* losses, float* lse, uint8_t* kinds, void* ws, unsigned* status, unsigned starve, void* stream) {
  const ssgd_status st = check_head(h, ldh, w, ldw, dtype, T, V, D, targets, ws, status);
  if (st != SSGD_OK || T == 0) return st;
  if (!losses || !lse || !kinds) return SSGD_ERR_NULL;
  if ((reinterpret_cast<uintptr_t>(losses) | reinterpret_cast<uintptr_t>(lse)) & 3u) return SSGD_ERR_ALIGN;
  DeviceInfo info;
  if (!device_info(&info)) return SSGD_ERR_CUDA;
  HeadSizes z;
  if (!head_sizes(T, V, D, info.sms, &z)) return SSGD_ERR_SIZE;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  return dtype == SSGD_BF16 ? head_forward(static_cast<const __nv_bfloat16*>(h), ldh, static_cast<const __nv_bfloat16*>(w), ldw, T, V, D, targets, ignore,
                                           losses, lse, kinds, ws, status, starve, info.sms, s)
                            : head_forward(static_cast<const __half*>(h), ldh, static_cast<const __half*>(w), ldw, T, V, D, targets, ignore, losses, lse,
                                           kinds, ws, status, starve, info.sms, s);
}

}  // namespace

extern "C" {

ssgd_status ssgd_xent_sizes(size_t T, size_t V, size_t D, size_t* forward_bytes, size_t* backward_bytes) {
  if (!forward_bytes || !backward_bytes) return SSGD_ERR_NULL;
  *forward_bytes = *backward_bytes = 16;
  if (T == 0 && V >= 1 && D >= 1) return SSGD_OK;
  DeviceInfo info;
  if (!device_info(&info)) return SSGD_ERR_CUDA;
  HeadSizes z;
  if (!head_sizes(T, V, D, info.sms, &z)) return SSGD_ERR_SIZE;
  *forward_bytes = z.forward_bytes;
  *backward_bytes = z.backward_bytes;
  return SSGD_OK;
}

ssgd_status ssgd_xent_align(const void* a, size_t lda, size_t step_a, size_t rows_a, void* to_a, const void* b, size_t ldb, size_t step_b, size_t rows_b,
                            void* to_b, size_t cols, size_t ldo, void* stream) {
  if (cols < 1 || cols > kSide || ldo < cols || ldo > 2 * kSide || rows_a > kSide || rows_b > kSide) return SSGD_ERR_SIZE;
  if ((rows_a && (!a || !to_a)) || (rows_b && (!b || !to_b))) return SSGD_ERR_NULL;
  if (ldo % 8 != 0 || !aligned16(to_a) || !aligned16(to_b) || ((reinterpret_cast<uintptr_t>(a) | reinterpret_cast<uintptr_t>(b)) & 1u)) return SSGD_ERR_ALIGN;
  const size_t blocks = ((rows_a + rows_b) * (ldo / 8) + 255) / 256;
  if (blocks > kMaxGrid) return SSGD_ERR_SIZE;
  if (blocks == 0) return SSGD_OK;
  const Scattered sa = {static_cast<const uint16_t*>(a), static_cast<uint16_t*>(to_a), lda, step_a, rows_a},
                  sb = {static_cast<const uint16_t*>(b), static_cast<uint16_t*>(to_b), ldb, step_b, rows_b};
  launch_kernel(xent_align_kernel, dim3((unsigned)blocks), dim3(256), 0, static_cast<cudaStream_t>(stream), true, sa, sb, (unsigned)cols, ldo);
  return launch_status();
}

ssgd_status ssgd_xent_forward(const void* h, size_t ldh, const void* w, size_t ldw, int dtype, size_t T, size_t V, size_t D, const int64_t* targets,
                              int64_t ignore, float* losses, float* lse, uint8_t* kinds, void* ws, unsigned* status, void* stream) {
  return checked_forward(h, ldh, w, ldw, dtype, T, V, D, targets, ignore, losses, lse, kinds, ws, status, 0, stream);
}

ssgd_status ssgd_xent_wait_selftest(const void* h, size_t ldh, const void* w, size_t ldw, int dtype, size_t T, size_t V, size_t D, const int64_t* targets,
                                    int64_t ignore, float* losses, float* lse, uint8_t* kinds, void* ws, unsigned* status, void* stream) {
  if (T > 256 || V > 256 || D > 128) return SSGD_ERR_SIZE;      // one round of tiles, two stages: the waits run out once
  return checked_forward(h, ldh, w, ldw, dtype, T, V, D, targets, ignore, losses, lse, kinds, ws, status, 16, stream);
}

ssgd_status ssgd_xent_backward(const void* h, size_t ldh, const void* w, size_t ldw, int dtype, size_t T, size_t V, size_t D, const int64_t* targets,
                               const float* lse, const uint8_t* kinds, const float* g, size_t g_stride, void* dh, size_t lddh, void* dw, int dw_type,
                               size_t lddw, void* ws, unsigned* status, void* stream) {
  const ssgd_status st = check_head(h, ldh, w, ldw, dtype, T, V, D, targets, ws, status);
  if (st != SSGD_OK) return st;
  if (dw && dtype_bytes((unsigned)dw_type) == 0) return SSGD_ERR_ARG;
  if ((dh && lddh < D) || (dw && (lddw < D || mul_overflows(V, lddw) || mul_overflows(V * lddw, 4)))) return SSGD_ERR_SIZE;
  if ((dh && (reinterpret_cast<uintptr_t>(dh) & 1u)) || (dw && reinterpret_cast<uintptr_t>(dw) % dtype_bytes((unsigned)dw_type) != 0)) return SSGD_ERR_ALIGN;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  if (T == 0) {
    if (!dw) return SSGD_OK;
    const size_t e = dtype_bytes((unsigned)dw_type);
    return cudaMemset2DAsync(dw, lddw * e, 0, D * e, V, s) == cudaSuccess ? SSGD_OK : SSGD_ERR_CUDA;
  }
  if (!lse || !kinds || !g) return SSGD_ERR_NULL;
  if ((reinterpret_cast<uintptr_t>(lse) | reinterpret_cast<uintptr_t>(g)) & 3u) return SSGD_ERR_ALIGN;
  if (!dh && !dw) return SSGD_OK;
  DeviceInfo info;
  if (!device_info(&info)) return SSGD_ERR_CUDA;
  const HeadBackward b = {h, w, ldh, ldw, T, V, D, targets, lse, kinds, g, g_stride, dh, lddh, dw, dw_type, lddw, static_cast<char*>(ws), status};
  return dtype == SSGD_BF16 ? head_backward<__nv_bfloat16>(b, info.sms, s) : head_backward<__half>(b, info.sms, s);
}

ssgd_status ssgd_xent_forward_block(const uint64_t* a) {
  if (!a) return SSGD_ERR_NULL;
  return ssgd_xent_forward(block_ptr<const void>(a[0]), a[1], block_ptr<const void>(a[2]), a[3], (int)a[4], a[5], a[6], a[7], block_ptr<const int64_t>(a[8]),
                           (int64_t)a[9], block_ptr<float>(a[10]), block_ptr<float>(a[11]), block_ptr<uint8_t>(a[12]), block_ptr<void>(a[13]),
                           block_ptr<unsigned>(a[14]), block_ptr<void>(a[15]));
}

ssgd_status ssgd_xent_backward_block(const uint64_t* a) {
  if (!a) return SSGD_ERR_NULL;
  return ssgd_xent_backward(block_ptr<const void>(a[0]), a[1], block_ptr<const void>(a[2]), a[3], (int)a[4], a[5], a[6], a[7], block_ptr<const int64_t>(a[8]),
                            block_ptr<const float>(a[9]), block_ptr<const uint8_t>(a[10]), block_ptr<const float>(a[11]), a[12], block_ptr<void>(a[13]), a[14],
                            block_ptr<void>(a[15]), (int)a[16], a[17], block_ptr<void>(a[18]), block_ptr<unsigned>(a[19]), block_ptr<void>(a[20]));
}

ssgd_status ssgd_xent_align_block(const uint64_t* a) {
  if (!a) return SSGD_ERR_NULL;
  return ssgd_xent_align(block_ptr<const void>(a[0]), a[1], a[2], a[3], block_ptr<void>(a[4]), block_ptr<const void>(a[5]), a[6], a[7], a[8],
                         block_ptr<void>(a[9]), a[10], a[11], block_ptr<void>(a[12]));
}

}  // extern "C"
