// Orthogonalised updates: a matrix U with its singular values brought near one by Newton-Schulz products (what the Muon optimiser
// does with its momentum), and the whole momentum step with it.  See include/signsgd.h for the contract.
//
//   X = U / |U|_F, then `steps` times  X <- a X + (b A + c A^2) X,  A = X X^T       (rows <= columns; else from the right)
//
// Three products a step, on the tensor cores, A and A^2 by the tiles on and above their diagonals alone.  Operands are fp16, and what a
// step loses, the next ones multiply by up to a (a direction whose singular value is still small grows by that), so the arithmetic is
// arranged to lose little.  X is kept as the sum of two fp16 matrices (22 bits).  With d = |X|_F^2 / s (s the shorter side) and A = d I + E
// the step is
//   X <- (a + b d + c d^2) X + ((b + 2 c d) E + c E^2) X:
// the part along X is done in fp32, and what goes through the products shrinks as X approaches its goal (A near I, E small).
//   TERMS = 3  products of both parts of each operand: error 4e-7 .. 2e-6 of the result, products in fp32 1e-6 .. 5e-6
//   TERMS = 1  products of the high parts: 4e-4 .. 1e-3, without d 2e-3 .. 3e-3; rounding to bf16 alone is 1.7e-3
// All matrices are stored times 2^13: elements are at most 1.2 in size, and the smallest that count stay normal numbers of fp16.

#include "half_product.cuh"

namespace {

constexpr float kScale = 8192.0f, kUnscale = 1.0f / 8192.0f;      // of X, E and M as they are stored

struct Polynomial { float a, b, c; };

// The 16-bit matrices that the products leave to one another, as boxes: high and low part.
struct Parts { CUtensorMap high, low; };
__device__ __forceinline__ void prefetch_parts(const Parts& p) {
  prefetch_tensor_map(&p.high);
  prefetch_tensor_map(&p.low);
}

// 32 neighbours of a row as two fp16 parts, two elements a word.
struct Words {
  unsigned high[16], low[16];
  __device__ __forceinline__ explicit Words(const float* v) {
#pragma unroll
    for (unsigned q = 0; q < 16; ++q) split_pair(v[2 * q], v[2 * q + 1], high[q], low[q]);
  }
};
// 32 x 32 elements as high and, LOW, low part.  What goes out takes the halves of a box in turn: one is written while the other is read.
template <bool LOW, bool ACROSS>
__device__ __forceinline__ void send_parts(const Box& box, unsigned offset, const Parts& to, unsigned x, unsigned y, unsigned matrix, const Words& w) {
  box.sent_but_last();
  if (ACROSS) box.put_words_across(offset, w.high);
  else box.put_words(offset, w.high);
  box.fence();
  box.send(to.high, offset, x, y, matrix);
  if (LOW) {
    box.sent_but_last();
    if (ACROSS) box.put_words_across(offset + 2048, w.low);
    else box.put_words(offset + 2048, w.low);
    box.fence();
    box.send(to.low, offset + 2048, x, y, matrix);
  }
}
// The same of a symmetric matrix: there, and, from tiles wholly above the diagonal, mirrored.  Tiles on the diagonal hold both halves
// themselves.
template <bool LOW>
__device__ __forceinline__ void send_symmetric(const Box& box, unsigned offset, const Parts& to, unsigned row0, unsigned column, unsigned matrix, bool mirrored,
                                               const float* v) {
  const Words w(v);
  send_parts<LOW, false>(box, offset, to, column, row0, matrix, w);
  if (mirrored) send_parts<LOW, true>(box, LOW ? offset : offset ^ 2048, to, row0, column, matrix, w);
}

// E = X X^T - d I.  d comes from the sums of squares that the last step left, added in a fixed order by each warp; the first tile of each
// matrix leaves it for the other two products.
template <bool LOW>
struct GramEpilogue {
  struct Args {
    Parts e;
    const float* squares;       // [matrix][count], or null: |X| is 1
    float* d;                   // [matrix]
    unsigned count, side;
  };
  static constexpr unsigned kBox = 4096;
  static __device__ __forceinline__ void prefetch(const Args& a) { prefetch_parts(a.e); }
  Box box;
  float d;
  unsigned row0, seen, matrix, half;
  bool mirrored;
  __device__ __forceinline__ GramEpilogue(const Args&, const Box& b) : box(b), seen(~0u), half(0) {}
  __device__ __forceinline__ void ahead(const Args&, unsigned) {}
  __device__ __forceinline__ void begin(const Args& a, const HalfPlace& at, unsigned first_row, unsigned) {
    row0 = first_row;
    matrix = at.matrix;
    mirrored = at.q0 >= at.p0 + at.rows;
    if (matrix != seen) {
      seen = matrix;
      float sum = 1.0f;
      if (a.squares) {
        sum = 0.0f;
        const float* from = a.squares + (size_t)matrix * a.count;
        for (unsigned i = box.lane; i < a.count; i += 16 * 32) {      // sixteen in flight: the products wait behind this
          float v[16];
#pragma unroll
          for (unsigned u = 0; u < 16; ++u) v[u] = i + u * 32 < a.count ? from[i + u * 32] : 0.0f;
#pragma unroll
          for (unsigned u = 0; u < 16; ++u) sum += v[u];
        }
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xFFFFFFFFu, sum, o);
      }
      d = sum / (float)a.side;
    }
    if (at.tile == 0 && row0 + box.lane == 0) a.d[matrix] = d;      // two warps: the same value
  }
  __device__ __forceinline__ void unit(const Args& a, unsigned column, unsigned, float (&v)[32]) {
    const unsigned on = row0 + box.lane - column;
#pragma unroll
    for (unsigned q = 0; q < 32; ++q) v[q] *= kUnscale;
    if (on < 32u) {
#pragma unroll
      for (unsigned q = 0; q < 32; ++q) v[q] = on == q ? v[q] - d * kScale : v[q];
    }
    send_symmetric<LOW>(box, half, a.e, row0, column, matrix, mirrored, v);
    if (!LOW && !mirrored) half ^= 2048;        // an odd number has gone out
  }
  __device__ __forceinline__ void end(const Args&, const HalfPlace&, unsigned) {}
  __device__ __forceinline__ void finish(const Args&) { box.finish(); }
};

// What an epilogue reads, 32 x 32 elements of two parts at a time, by one or two boxes in which what it makes of them goes out again.  With two
// the next is asked for before the last is taken; with one (where shared memory holds no more beside stages of three terms and 256
// columns) when the last has gone, which the products that run on meanwhile hide.
template <unsigned BOXES>
struct Reader {
  unsigned asks = 0, takes = 0, later = ~0u;    // later: a column that has to wait for the box
  __device__ __forceinline__ void ask(Box& box, const CUtensorMap& high, const CUtensorMap* low, unsigned column, unsigned row, unsigned matrix) {
    if (BOXES == 1 && asks != takes) {
      later = column;
      return;
    }
    box.sent();
    const unsigned b = BOXES == 1 ? 0 : asks & 1u;
    box.ask(b, b * 4096, high, low, column, row, matrix);
    ++asks;
  }
  // Where the elements are; for one box it is taken until `done`.
  __device__ __forceinline__ unsigned take(Box& box) {
    const unsigned b = BOXES == 1 ? 0 : takes & 1u;
    box.take(b);
    if (BOXES == 2) ++takes;
    return b * 4096;
  }
  __device__ __forceinline__ void done(Box& box, const CUtensorMap& high, const CUtensorMap* low, unsigned row, unsigned matrix) {
    if (BOXES == 1) {
      ++takes;
      if (later != ~0u) {
        const unsigned column = later;
        later = ~0u;
        ask(box, high, low, column, row, matrix);
      }
    }
  }
};

// M = p E + c E^2, p = b + 2 c d.
struct PolynomialArgs {
  Parts e, m;
  const float* d;
  Polynomial f;
};
template <bool LOW, unsigned BOXES>
struct PolynomialEpilogue {
  using Args = PolynomialArgs;
  static constexpr unsigned kBox = BOXES * 4096;
  static __device__ __forceinline__ void prefetch(const Args& a) {
    prefetch_parts(a.m);
    prefetch_parts(a.e);
  }
  Box box;
  Reader<BOXES> reader;
  float p;
  unsigned row0, matrix;
  bool mirrored;
  __device__ __forceinline__ PolynomialEpilogue(const Args&, const Box& b) : box(b) {}
  __device__ __forceinline__ void begin(const Args& a, const HalfPlace& at, unsigned first_row, unsigned) {
    row0 = first_row;
    matrix = at.matrix;
    mirrored = at.q0 >= at.p0 + at.rows;
    p = a.f.b + 2.0f * a.f.c * a.d[matrix];
  }
  __device__ __forceinline__ void ahead(const Args& a, unsigned column) { reader.ask(box, a.e.high, LOW ? &a.e.low : nullptr, column, row0, matrix); }
  __device__ __forceinline__ void unit(const Args& a, unsigned column, unsigned, float (&v)[32]) {
    const float c = a.f.c * kUnscale;
    const unsigned from = reader.take(box);
#pragma unroll
    for (unsigned q = 0; q < 4; ++q) {
      float e[8];
      box.get8(from, q, e);
      if (LOW) {
        float low[8];
        box.get8(from + 2048, q, low);
#pragma unroll
        for (unsigned i = 0; i < 8; ++i) e[i] += low[i];
      }
#pragma unroll
      for (unsigned i = 0; i < 8; ++i) v[8 * q + i] = fmaf(c, v[8 * q + i], p * e[i]);
    }
    __syncwarp();
    send_symmetric<LOW>(box, from, a.m, row0, column, matrix, mirrored, v);
    reader.done(box, a.e.high, LOW ? &a.e.low : nullptr, row0, matrix);
  }
  __device__ __forceinline__ void end(const Args&, const HalfPlace&, unsigned) {}
  __device__ __forceinline__ void finish(const Args&) { box.finish(); }
};

// X' = q X + M X, q = a + b d + c d^2: kept for the next step, with its sum of squares; or, behind the last, written out as T; or
// x <- x - delta X'.
enum UpdateTo { kNextStep, kOut, kParameters };
template <typename T>
struct UpdateArgs {
  Parts x, next;
  const float* d;
  float* squares;               // [matrix][count]
  T* out;
  size_t ldo, out_stride;
  Polynomial f;
  float delta;
  unsigned rows, count, slots;          // sums of squares of a matrix, and of a tile
};
template <int TO, typename T, unsigned BOXES>
struct UpdateEpilogue {
  using Args = UpdateArgs<T>;
  static constexpr unsigned kBox = BOXES * 4096;
  static __device__ __forceinline__ void prefetch(const Args& a) {
    if (TO == kNextStep) prefetch_parts(a.next);
    prefetch_parts(a.x);
  }
  Box box;
  Reader<BOXES> reader;
  float q, sum;
  unsigned row0, matrix;
  __device__ __forceinline__ UpdateEpilogue(const Args&, const Box& b) : box(b) {}
  __device__ __forceinline__ void begin(const Args& a, const HalfPlace& at, unsigned first_row, unsigned) {
    row0 = first_row;
    matrix = at.matrix;
    const float d = a.d[matrix];
    q = a.f.a + d * (a.f.b + d * a.f.c);
    sum = 0.0f;
  }
  __device__ __forceinline__ void ahead(const Args& a, unsigned column) { reader.ask(box, a.x.high, &a.x.low, column, row0, matrix); }
  __device__ __forceinline__ void unit(const Args& a, unsigned column, unsigned left, float (&v)[32]) {
    const unsigned from = reader.take(box);
#pragma unroll
    for (unsigned p = 0; p < 4; ++p) {
      float high[8], low[8];
      box.get8(from, p, high);
      box.get8(from + 2048, p, low);
#pragma unroll
      for (unsigned i = 0; i < 8; ++i) v[8 * p + i] = fmaf(q, high[i] + low[i], v[8 * p + i] * kUnscale);
    }
    __syncwarp();
    if constexpr (TO == kNextStep) {
      if (row0 + box.lane < a.rows) {           // behind the last column there are zeros
#pragma unroll
        for (unsigned i = 0; i < 32; ++i) sum = fmaf(v[i], v[i], sum);
      }
      send_parts<true, false>(box, from, a.next, column, row0, matrix, Words(v));
    } else {
      const float by = TO == kOut ? kUnscale : -a.delta * kUnscale;
#pragma unroll
      for (unsigned i = 0; i < 32; ++i) v[i] *= by;
      const Box whole(box.at + from, box.full, box.lane);
      T* o = a.out + matrix * a.out_stride + (size_t)row0 * a.ldo + column;
      const unsigned rows = min(32u, a.rows - row0);
      if constexpr (TO == kOut) whole.rows_out(o, a.ldo, rows, left, v);
      else whole.rows_join(o, a.ldo, o, a.ldo, rows, left, v, [](float x, float step) { return x + step; });
      box.fence();                              // the threads' own writes come before the copy that is asked for next into the same bytes
    }
    reader.done(box, a.x.high, &a.x.low, row0, matrix);
  }
  __device__ __forceinline__ void end(const Args& a, const HalfPlace& at, unsigned warp) {
    if constexpr (TO == kNextStep) {
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xFFFFFFFFu, sum, o);
      if (box.lane == 0) a.squares[(size_t)matrix * a.count + at.tile * a.slots + warp] = sum * (kUnscale * kUnscale);
    }
  }
  __device__ __forceinline__ void finish(const Args&) { box.finish(); }
};

// ---------------------------------------------------------------------------------------------------------------------
// Before the products: the norm, then X's two parts.  A momentum step makes its U on the way, in both passes the same:
//   m <- fma(beta, m, fl((1 - beta) g)),  u = m, or looking ahead fma(beta, m, fl((1 - beta) g))

struct Whole {                    // a batch of matrices, high and low part
  __half *high, *low;
  size_t ld, stride;
};

struct Source {
  const void* u;                // the matrix itself; with a momentum the gradient
  float* m;
  size_t ldu, u_stride, ldm, m_stride;
  float beta;
  unsigned rows, cols;
  bool ahead, eights;           // eights: every row of u and m can be read 16 bytes at a time, eight elements from its start on
};
enum { kPlainSource, kMomentum };

// Eight elements of a row as they lie in memory, `left` of them inside, zeros behind; and their values.
template <typename T>
struct Eight { uint4 q[sizeof(T) / 2]; };
template <typename T>
__device__ __forceinline__ void source_load(const T* p, unsigned left, bool eights, Eight<T>& e) {
  if (eights && left >= 8) {
#pragma unroll
    for (unsigned i = 0; i < sizeof(T) / 2; ++i) e.q[i] = reinterpret_cast<const uint4*>(p)[i];
  } else {
    unsigned w[2 * sizeof(T)];
    if constexpr (sizeof(T) == 4) {
#pragma unroll
      for (unsigned i = 0; i < 8; ++i) w[i] = i < left ? __float_as_uint(p[i]) : 0u;
    } else {
      const unsigned short* h = reinterpret_cast<const unsigned short*>(p);
#pragma unroll
      for (unsigned i = 0; i < 4; ++i) w[i] = (2 * i < left ? h[2 * i] : 0u) | (2 * i + 1 < left ? (unsigned)h[2 * i + 1] << 16 : 0u);
    }
#pragma unroll
    for (unsigned i = 0; i < sizeof(T) / 2; ++i) e.q[i] = make_uint4(w[4 * i], w[4 * i + 1], w[4 * i + 2], w[4 * i + 3]);
  }
}
template <typename T>
__device__ __forceinline__ void eight_values(const Eight<T>& e, float (&v)[8]) {
  if constexpr (sizeof(T) == 4) {
#pragma unroll
    for (unsigned i = 0; i < 2; ++i) {
      v[4 * i] = __uint_as_float(e.q[i].x); v[4 * i + 1] = __uint_as_float(e.q[i].y);
      v[4 * i + 2] = __uint_as_float(e.q[i].z); v[4 * i + 3] = __uint_as_float(e.q[i].w);
    }
  } else {
    v[0] = low_to_float(T(), e.q[0].x); v[1] = high_to_float(T(), e.q[0].x); v[2] = low_to_float(T(), e.q[0].y); v[3] = high_to_float(T(), e.q[0].y);
    v[4] = low_to_float(T(), e.q[0].z); v[5] = high_to_float(T(), e.q[0].z); v[6] = low_to_float(T(), e.q[0].w); v[7] = high_to_float(T(), e.q[0].w);
  }
}

// U at eight columns of a row, in two halves, so that several can be on their way; FIRST: m is brought forward and written.
template <typename T>
struct Fetched {
  Eight<float> m;
  Eight<T> g;
};
template <int KIND, bool FIRST, typename T>
__device__ __forceinline__ void source_fetch(const Source& s, size_t matrix, unsigned row, unsigned column, Fetched<T>& f) {
  const unsigned left = s.cols - column;
  if (KIND == kMomentum) source_load(s.m + matrix * s.m_stride + (size_t)row * s.ldm + column, left, s.eights, f.m);
  if (KIND == kPlainSource || FIRST || s.ahead) source_load(static_cast<const T*>(s.u) + matrix * s.u_stride + (size_t)row * s.ldu + column, left, s.eights, f.g);
}
template <int KIND, bool FIRST, typename T>
__device__ __forceinline__ void source_values(const Source& s, size_t matrix, unsigned row, unsigned column, const Fetched<T>& f, float (&u)[8]) {
  if constexpr (KIND == kPlainSource) {
    eight_values(f.g, u);
  } else {
    float m[8], g[8];
    eight_values(f.m, m);
    if (FIRST || s.ahead) {
      eight_values(f.g, g);
#pragma unroll
      for (unsigned i = 0; i < 8; ++i) g[i] = __fmul_rn(1.0f - s.beta, g[i]);
    }
    if (FIRST) {
      float* mp = s.m + matrix * s.m_stride + (size_t)row * s.ldm + column;
      const unsigned left = s.cols - column;
#pragma unroll
      for (unsigned i = 0; i < 8; ++i) m[i] = __fmaf_rn(s.beta, m[i], g[i]);
      if (s.eights && left >= 8) {
        *reinterpret_cast<float4*>(mp) = make_float4(m[0], m[1], m[2], m[3]);
        *reinterpret_cast<float4*>(mp + 4) = make_float4(m[4], m[5], m[6], m[7]);
      } else {
#pragma unroll
        for (unsigned i = 0; i < 8; ++i)
          if (i < left) mp[i] = m[i];
      }
    }
#pragma unroll
    for (unsigned i = 0; i < 8; ++i) u[i] = s.ahead ? __fmaf_rn(s.beta, m[i], g[i]) : m[i];
  }
}

constexpr unsigned kNormThreads = 256;

// f(row, column, U's eight values) for this CTA's share of a matrix, BATCH loads of each array in flight.  What lies behind a row's last
// column is zero.
template <int KIND, bool FIRST, typename T, typename F>
__device__ __forceinline__ void each_eight(const Source& s, size_t matrix, F f) {
  constexpr unsigned kBatch = KIND == kMomentum ? 2 : sizeof(T) == 2 ? 8 : 4;
  const unsigned eights = (s.cols + 7) / 8, total = eights * s.rows, step = gridDim.x * kNormThreads;
  for (unsigned i0 = blockIdx.x * kNormThreads + threadIdx.x; i0 < total; i0 += kBatch * step) {
    Fetched<T> v[kBatch];
    unsigned row[kBatch];
#pragma unroll
    for (unsigned b = 0; b < kBatch; ++b) {
      const unsigned i = i0 + b * step;
      row[b] = i / eights;
      if (i < total) source_fetch<KIND, FIRST, T>(s, matrix, row[b], (i - row[b] * eights) * 8, v[b]);
    }
#pragma unroll
    for (unsigned b = 0; b < kBatch; ++b) {
      const unsigned i = i0 + b * step;
      if (i >= total) break;
      const unsigned column = (i - row[b] * eights) * 8;
      float u[8];
      source_values<KIND, FIRST, T>(s, matrix, row[b], column, v[b], u);
      f(row[b], column, u);
    }
  }
}

template <int KIND, typename T>
__global__ void __launch_bounds__(kNormThreads)
orthogonal_norm_kernel(const Source s, double* __restrict__ partial) {
  __shared__ double part[kNormThreads / 32];
  pdl_launch_dependents();
  pdl_wait();
  double sum = 0.0;
  each_eight<KIND, true, T>(s, blockIdx.y, [&](unsigned, unsigned column, const float (&u)[8]) {
#pragma unroll
    for (unsigned k = 0; k < 8; ++k)
      if (column + k < s.cols) sum = fma((double)u[k], (double)u[k], sum);
  });
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xFFFFFFFFu, sum, o);
  if ((threadIdx.x & 31u) == 0) part[threadIdx.x >> 5] = sum;
  __syncthreads();
  if (threadIdx.x == 0) {
    for (unsigned w = 1; w < kNormThreads / 32; ++w) sum += part[w];
    partial[(size_t)blockIdx.y * gridDim.x + blockIdx.x] = sum;
  }
}

// scale / norm in two factors, a power of two that brings the norm to [1, 2) where that is an fp32 number, and the rest: the first
// multiplication is exact, and neither leaves fp32's range.  A zero matrix stays zero, one that is not finite becomes NaN.
struct Inverse { float first, rest; };
__device__ __forceinline__ Inverse inverse_of(double norm, float scale) {
  const bool finite = isfinite(norm);
  const int e = norm > 0.0 && finite ? max(-126, min(126, -ilogb(norm))) : 0;
  const float first = __uint_as_float((unsigned)(127 + e) << 23);
  return {first, norm > 0.0 ? (finite ? (float)((double)scale / (norm * (double)first)) : __uint_as_float(0x7FC00000u)) : finite ? 0.0f : __uint_as_float(0x7FC00000u)};
}

template <int KIND, typename T>
__global__ void __launch_bounds__(kNormThreads)
orthogonal_split_kernel(const Source s, const double* __restrict__ partial, unsigned parts, const Whole x) {
  __shared__ double norm2;
  pdl_launch_dependents();
  pdl_wait();
  if (threadIdx.x < 32) {
    double sum = 0.0;
    for (unsigned i = threadIdx.x; i < parts; i += 32) sum += partial[(size_t)blockIdx.y * parts + i];
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xFFFFFFFFu, sum, o);
    if (threadIdx.x == 0) norm2 = sum;
  }
  __syncthreads();
  const Inverse inverse = inverse_of(sqrt(norm2), kScale);
  each_eight<KIND, false, T>(s, blockIdx.y, [&](unsigned row, unsigned column, const float (&u)[8]) {
    unsigned high[4], low[4];
#pragma unroll
    for (unsigned k = 0; k < 4; ++k)
      split_pair(u[2 * k] * inverse.first * inverse.rest, u[2 * k + 1] * inverse.first * inverse.rest, high[k], low[k]);
    const size_t at = blockIdx.y * x.stride + (size_t)row * x.ld + column;
    *reinterpret_cast<uint4*>(x.high + at) = make_uint4(high[0], high[1], high[2], high[3]);
    *reinterpret_cast<uint4*>(x.low + at) = make_uint4(low[0], low[1], low[2], low[3]);
  });
}

// ---------------------------------------------------------------------------------------------------------------------
// Matrices of up to 128 x 128: a CTA does all of it, one launch instead of two and three a step (64 x 64, five steps: 80 -> 22 us).
//
// X and E = X X^T - d I stay in registers in fp32, a thread a row and 32 columns, which is how the tensor cores give their sums back; their
// fp16 parts lie in shared memory as the tensor cores take operands, 64 columns to a block of 128 rows x 128 bytes.  The same
// bytes serve as an operand with its k side by side and as one with its rows side by side: X X^T and M X, and for tall matrices X^T X
// and X M, need no transpose.  M takes E's place.

constexpr unsigned kSmallSide = 128, kSmallThreads = 512;
constexpr unsigned kSmallPart = 32768;                                      // one 128 x 128 fp16 matrix
constexpr unsigned kStageLd = kSmallSide + 1;                               // fp32 rows on their way in and out
constexpr unsigned kSmallSmem = 4 * kSmallPart + kSmallSide * kStageLd * 4 + 1024;

struct SmallArgs {
  Source source;
  int source_type, out_type, momentum;
  void* out;                    // of out_type, or the parameters
  size_t ldo, out_stride;
  Polynomial f;
  float delta;
  unsigned steps, starve;
  unsigned* status;
};

__device__ __forceinline__ float load_any(const void* p, int type, size_t at) {
  switch (type) {
    case SSGD_F32: return static_cast<const float*>(p)[at];
    case SSGD_BF16: return to_float(static_cast<const __nv_bfloat16*>(p)[at]);
    default: return to_float(static_cast<const __half*>(p)[at]);
  }
}
__device__ __forceinline__ void store_any(void* p, int type, size_t at, float v) {
  switch (type) {
    case SSGD_F32: static_cast<float*>(p)[at] = v; break;
    case SSGD_BF16: static_cast<__nv_bfloat16*>(p)[at] = from_float<__nv_bfloat16>(v); break;
    default: static_cast<__half*>(p)[at] = from_float<__half>(v); break;
  }
}

// A thread's 32 values of a row as the two parts of an operand; group: which 32 columns.
__device__ __forceinline__ void put_operand(unsigned high, unsigned row, unsigned group, const float (&v)[32]) {
  const unsigned block = high + group / 2 * (kSmallPart / 2) + row * 128;
#pragma unroll
  for (unsigned q = 0; q < 4; ++q) {
    unsigned h[4], l[4];
#pragma unroll
    for (unsigned i = 0; i < 4; ++i) split_pair(v[8 * q + 2 * i], v[8 * q + 2 * i + 1], h[i], l[i]);
    const unsigned at = block + ((((group & 1u) * 4 + q) ^ (row & 7u)) << 4);
    store_shared16(at, h[0], h[1], h[2], h[3]);
    store_shared16(at + kSmallPart, l[0], l[1], l[2], l[3]);
  }
}

// D = P Q^T of operands in shared memory, k in pieces of 16; by one thread.  Unrolled, with descriptors that differ by constants: what the
// thread computes between two of them is what the tensor cores wait for.
template <bool P_BY_ROWS, bool Q_BY_ROWS>
__device__ __forceinline__ void small_product(unsigned d, unsigned p, unsigned q, unsigned columns, unsigned k, unsigned done) {
  const unsigned idesc = mma_half_descriptor(128, (columns + 15) / 16 * 16, false, P_BY_ROWS, Q_BY_ROWS);
  const uint64_t pd = half_descriptor(p, P_BY_ROWS, kSmallPart / 2), qd = half_descriptor(q, Q_BY_ROWS, kSmallPart / 2);
  constexpr unsigned low = kSmallPart >> 4;
  // rows side by side: 16 of k are 16 rows; else 32 bytes, four of them a block
  auto at = [](bool by_rows, unsigned c) { return by_rows ? c * (2048 >> 4) : c / 4 * (kSmallPart / 2 >> 4) + c % 4 * (32 >> 4); };
#pragma unroll
  for (unsigned c = 0; c < kSmallSide / 16; ++c) {
    if (c == 0 || c * 16 < k) {
      mma_half<false>(d, pd + at(P_BY_ROWS, c), qd + at(Q_BY_ROWS, c) + low, idesc, c > 0);
      mma_half<false>(d, pd + at(P_BY_ROWS, c) + low, qd + at(Q_BY_ROWS, c), idesc, true);
    }
  }
#pragma unroll
  for (unsigned c = 0; c < kSmallSide / 16; ++c)
    if (c == 0 || c * 16 < k) mma_half<false>(d, pd + at(P_BY_ROWS, c), qd + at(Q_BY_ROWS, c), idesc, true);
  tcgen05_commit(done);
}

__global__ void __launch_bounds__(kSmallThreads, 1)
orthogonal_small_kernel(const SmallArgs a) {
  extern __shared__ unsigned char small_smem[];
  __shared__ __align__(8) uint64_t done_bar;
  __shared__ unsigned tmem_base;
  __shared__ double norms[kSmallThreads / 32];
  __shared__ float squares[kSmallThreads / 32];
  __shared__ Inverse inverse;
  const unsigned pad = (1024u - (smem_u32(small_smem) & 1023u)) & 1023u;
  const unsigned x_at = smem_u32(small_smem) + pad, e_at = x_at + 2 * kSmallPart;
  float* stage = reinterpret_cast<float*>(small_smem + pad + 4 * kSmallPart);
  const unsigned warp = threadIdx.x >> 5, lane = threadIdx.x & 31u, row = (warp & 3u) * 32 + lane, group = warp >> 2;
  const unsigned rows = a.source.rows, cols = a.source.cols, side = min(rows, cols), matrix = blockIdx.x;
  const unsigned done = smem_u32(&done_bar);
  const bool tall = rows > cols;

  if (threadIdx.x == 0) {
    mbarrier_init(done, a.starve ? 2 : 1);
    mbarrier_init_fence();
  }
  pdl_launch_dependents();
  pdl_wait();                                   // before tensor memory is taken: its last holder has finished
  if (warp == 1) tmem_alloc(smem_u32(&tmem_base), 128);
  tcgen05_fence_before();

  // U, a warp a row, lanes side by side, two rows in flight; a momentum is brought forward on the way.
  const size_t u0 = matrix * a.source.u_stride, m0 = matrix * a.source.m_stride;
  constexpr unsigned kWarps = kSmallThreads / 32;
  for (unsigned r0 = warp; r0 < rows; r0 += 2 * kWarps) {
    float u[8], m[8];
#pragma unroll
    for (unsigned k = 0; k < 8; ++k) {
      const unsigned r = r0 + k / 4 * kWarps, c = lane + k % 4 * 32;
      u[k] = m[k] = 0.0f;
      if (r < rows && c < cols) {
        u[k] = load_any(a.source.u, a.source_type, u0 + (size_t)r * a.source.ldu + c);
        if (a.momentum) m[k] = a.source.m[m0 + (size_t)r * a.source.ldm + c];
      }
    }
#pragma unroll
    for (unsigned k = 0; k < 8; ++k) {
      const unsigned r = r0 + k / 4 * kWarps, c = lane + k % 4 * 32;
      if (r < rows && c < cols) {
        if (a.momentum) {
          const float g = __fmul_rn(1.0f - a.source.beta, u[k]), next = __fmaf_rn(a.source.beta, m[k], g);
          a.source.m[m0 + (size_t)r * a.source.ldm + c] = next;
          u[k] = a.source.ahead ? __fmaf_rn(a.source.beta, next, g) : next;
        }
        stage[r * kStageLd + c] = u[k];
      }
    }
  }
  __syncthreads();
  tcgen05_fence_after();
  const unsigned tmem = tmem_base, lanes = tmem + ((warp & 3u) << 21) + group * 32;

  // Where a warp has something of X (of E, M): the others only keep step.  What lies beyond a matrix is zero, and stays so.
  const unsigned row0 = (warp & 3u) * 32;
  const bool has_x = row0 < rows && group * 32 < cols, has_e = row0 < side && group * 32 < side;
  float x[32], e[32];                           // times 2^13, as their parts are stored
  double sum = 0.0;
#pragma unroll
  for (unsigned q = 0; q < 32; ++q) x[q] = e[q] = 0.0f;
  if (has_x) {
#pragma unroll
    for (unsigned q = 0; q < 32; ++q) x[q] = row < rows && group * 32 + q < cols ? stage[row * kStageLd + group * 32 + q] : 0.0f;
#pragma unroll
    for (unsigned q = 0; q < 32; ++q) sum = fma((double)x[q], (double)x[q], sum);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xFFFFFFFFu, sum, o);
  }
  if (lane == 0) norms[warp] = sum;
  __syncthreads();
  if (warp == 0) {
    sum = lane < kWarps ? norms[lane] : 0.0;
#pragma unroll
    for (int o = 8; o > 0; o >>= 1) sum += __shfl_xor_sync(0xFFFFFFFFu, sum, o);
    if (lane == 0) inverse = inverse_of(sqrt(sum), kScale);
  }
  __syncthreads();
  if (has_x) {
    const Inverse by = inverse;
#pragma unroll
    for (unsigned q = 0; q < 32; ++q) x[q] = x[q] * by.first * by.rest;
  }
  put_operand(x_at, row, group, x);
  put_operand(e_at, row, group, e);
  async_proxy_fence();
  __syncthreads();

  bool ok = true;
  unsigned parity = 0;
  float d = 1.0f / (float)side;
  // The tensor cores' sums are there, for every thread or for none.  One warp asks; the others wait for it at the CTA's barrier.
  auto wait = [&]() {
    bool there = true;
    if (warp == 0) {
      there = false;
      for (unsigned i = 0; i < 16 * kHalfPolls && !there; ++i) there = mbarrier_test(done, parity);
    }
    ok = __syncthreads_and(there) != 0;
    parity ^= 1u;
    tcgen05_fence_after();
    return ok;
  };
  // Operands as the threads have written them are the tensor cores' to read, and the sums that the threads have read theirs to write.
  auto publish = [&]() {
    async_proxy_fence();
    tcgen05_fence_before();
    __syncthreads();
    tcgen05_fence_after();
  };
  // This warp's sums, times 2^13.  The product has had `columns`, rounded up to 16: behind them tensor memory holds anything.
  auto sums = [&](unsigned columns, float (&v)[32]) {
    unsigned u[32];
    tmem_read32(lanes, u);
    const bool second = group * 32 + 16 < columns;
#pragma unroll
    for (unsigned q = 0; q < 32; ++q) v[q] = q < 16 || second ? __uint_as_float(u[q]) * kUnscale : 0.0f;
  };
  for (unsigned k = 0; k < a.steps; ++k) {
    if (warp == 0 && elect_one()) {
      if (tall) small_product<true, true>(tmem, x_at, x_at, cols, rows, done);
      else small_product<false, false>(tmem, x_at, x_at, rows, cols, done);
    }
    __syncwarp();
    if (!wait()) break;
    if (has_e) {
      sums(side, e);
      if (row0 == group * 32 && row < side) {
#pragma unroll
        for (unsigned q = 0; q < 32; ++q) e[q] = lane == q ? e[q] - d * kScale : e[q];
      }
      put_operand(e_at, row, group, e);
    }
    publish();
    if (warp == 0 && elect_one()) small_product<false, false>(tmem, e_at, e_at, side, side, done);
    __syncwarp();
    if (!wait()) break;
    const float p = a.f.b + 2.0f * a.f.c * d, own = a.f.a + d * (a.f.b + d * a.f.c);
    if (has_e) {
      float v[32];
      sums(side, v);
#pragma unroll
      for (unsigned q = 0; q < 32; ++q) e[q] = fmaf(a.f.c, v[q], p * e[q]);
      put_operand(e_at, row, group, e);
    }
    publish();
    if (warp == 0 && elect_one()) {
      if (tall) small_product<false, false>(tmem, x_at, e_at, cols, cols, done);
      else small_product<false, true>(tmem, e_at, x_at, cols, rows, done);
    }
    __syncwarp();
    if (!wait()) break;
    float square = 0.0f;
    if (has_x) {
      float v[32];
      sums(cols, v);
#pragma unroll
      for (unsigned q = 0; q < 32; ++q) {
        x[q] = fmaf(own, x[q], v[q]);
        square = fmaf(x[q], x[q], square);
      }
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) square += __shfl_xor_sync(0xFFFFFFFFu, square, o);
    }
    if (k + 1 == a.steps) break;
    if (lane == 0) squares[warp] = square;
    if (has_x) put_operand(x_at, row, group, x);
    publish();
    d = 0.0f;
#pragma unroll
    for (unsigned w = 0; w < kWarps; ++w) d += squares[w];
    d *= kUnscale * kUnscale / (float)side;
  }

  if (ok) {
    if (has_x) {
#pragma unroll
      for (unsigned q = 0; q < 32; ++q) stage[row * kStageLd + group * 32 + q] = x[q] * kUnscale;
    }
    tcgen05_fence_before();
    __syncthreads();
    const size_t o0 = matrix * a.out_stride;
    for (unsigned r0 = warp; r0 < rows; r0 += 2 * kWarps) {
      float old[8];
#pragma unroll
      for (unsigned k = 0; k < 8; ++k) {
        const unsigned r = r0 + k / 4 * kWarps, c = lane + k % 4 * 32;
        old[k] = a.momentum && r < rows && c < cols ? static_cast<const float*>(a.out)[o0 + (size_t)r * a.ldo + c] : 0.0f;
      }
#pragma unroll
      for (unsigned k = 0; k < 8; ++k) {
        const unsigned r = r0 + k / 4 * kWarps, c = lane + k % 4 * 32;
        if (r < rows && c < cols) {
          const float v = stage[r * kStageLd + c];
          store_any(a.out, a.out_type, o0 + (size_t)r * a.ldo + c, a.momentum ? fmaf(-a.delta, v, old[k]) : v);
        }
      }
    }
  } else {
    if (threadIdx.x == 0) atomicOr(a.status, 1u);
    __syncthreads();
  }
  if (warp == 1) {
    tcgen05_fence_after();
    tmem_free(tmem, 128);
  }
}

// ---------------------------------------------------------------------------------------------------------------------
// Matrices of a few tiles: a cluster of CTAs does all steps of one matrix in one launch, a barrier of the cluster between two products.  (A
// launch of its own costs a small product 4 of its 6 us: the gap, the start, code that is cold.)  Tiles of 128 x 64 and the same
// stages, sums and epilogues as half_product_kernel's; what one product leaves for the next goes through L2.

template <int TO, typename T>
struct ClusterArgs {
  CUtensorMap x[2][2], e[2], m[2];              // operands in boxes of 64 x 64, high and low part; the same boxes serve either way round
  typename GramEpilogue<true>::Args gram[2];          // of the first step, and of the others
  PolynomialArgs polynomial;
  UpdateArgs<float> next[2];
  UpdateArgs<T> last;
  unsigned rows, cols, steps, starve;
  unsigned* status;
};

// Stages between two times that a sum of three terms is taken.  Tiles of 256 columns have two sums on their way and 128 a thread to add: four
// times as many there (steps of 24 x 1024 x 1024: 4 stages 2.12 ms, 8 1.94, of 8192 x 2048 1.66 and 1.59; error 7e-7 and 1.6e-6 of the result, products
// in fp32 3.1e-6).
constexpr int kChunk = 2;
using ClusterShape = HalfShape<false, 64, 3, kChunk, 8192>;

struct ClusterState {
  unsigned stage0, full, empty, acc_full, acc_free, tmem, warp, lane, rank, size, matrix, starve;
  unsigned n, t;                                // stages and sums so far, as this thread's role counts them
  unsigned phase;                               // of this warp's box: the epilogues share it
  bool ok;
};

// One product, tile after tile by the CTAs of the cluster in turn.
template <int LAYOUT, class Epilogue>
__device__ __forceinline__ void cluster_product(ClusterState& st, bool symmetric, const CUtensorMap* p_maps, const CUtensorMap* q_maps, unsigned P, unsigned Q, unsigned K,
                                                Epilogue& epilogue, const typename Epilogue::Args& args) {
  using S = ClusterShape;
  constexpr unsigned low = (S::p_bytes + S::q_bytes) >> 4;
  const unsigned tiles_p = (P + 127) / 128, tiles_q = (Q + 63) / 64, stages = (K + 63) / 64, chunks = (K + 15) / 16;
  // f(first row, first column) for this CTA's tiles, along the rows of tiles, in a symmetric product from the diagonal on
  auto each_tile = [&](auto f) {
    unsigned tile = st.rank;
    for (unsigned i = 0; i < tiles_p && st.ok; ++i) {
      const unsigned begin = symmetric ? 2 * i : 0, count = tiles_q > begin ? tiles_q - begin : 0;
      for (; tile < count && st.ok; tile += st.size) f(i * 128, (begin + tile) * 64);
      tile -= min(tile, count);
    }
  };
  if (st.warp == 0) {
    if (elect_one()) {
      each_tile([&](unsigned p0, unsigned q0) {
        for (unsigned k = 0; k < stages; ++k, ++st.n) {
          const unsigned s = st.n % S::stages;
          if (st.n >= S::stages) st.ok = mbarrier_wait(st.empty + 8 * s, (st.n / S::stages - 1) & 1u, kHalfPolls);
          if (!st.ok) break;
          const unsigned base = st.stage0 + s * S::stage_bytes, bar = st.full + 8 * s;
          mbarrier_expect(bar, 2 * (S::p_bytes + S::q_bytes) + st.starve);
#pragma unroll
          for (unsigned h = 0; h < 2; ++h) {
            const unsigned pd = base + h * (S::p_bytes + S::q_bytes), qd = pd + S::p_bytes;
#pragma unroll
            for (unsigned j = 0; j < 2; ++j) {
              if (LAYOUT & 2) tma_load_3d(pd + j * 8192, &p_maps[h], (int)(p0 + 64 * j), (int)(k * 64), (int)st.matrix, bar);
              else tma_load_3d(pd + j * 8192, &p_maps[h], (int)(k * 64), (int)(p0 + 64 * j), (int)st.matrix, bar);
            }
            if (LAYOUT & 1) tma_load_3d(qd, &q_maps[h], (int)q0, (int)(k * 64), (int)st.matrix, bar);
            else tma_load_3d(qd, &q_maps[h], (int)(k * 64), (int)q0, (int)st.matrix, bar);
          }
        }
      });
    }
    __syncwarp();
  } else if (st.warp == 1) {
    if (elect_one()) {
      const uint64_t p_desc = half_descriptor(st.stage0, (LAYOUT & 2) != 0), q_desc = half_descriptor(st.stage0 + S::p_bytes, (LAYOUT & 1) != 0);
      const unsigned idesc = mma_half_descriptor(128, 64, false, (LAYOUT & 2) != 0, (LAYOUT & 1) != 0);
      each_tile([&](unsigned, unsigned) {
        for (unsigned k = 0; k < stages; ++k, ++st.n) {
          const unsigned s = st.n % S::stages, acc = st.t % S::accs;
          const bool fresh = k % kChunk == 0, taken = k % kChunk == kChunk - 1 || k + 1 == stages;
          if (fresh && st.t >= S::accs) st.ok = mbarrier_wait(st.acc_free + 8 * acc, (st.t / S::accs - 1) & 1u, kHalfPolls);
          st.ok = st.ok && mbarrier_wait(st.full + 8 * s, (st.n / S::stages) & 1u, kHalfPolls);
          if (!st.ok) break;
          tcgen05_fence_after();
          const unsigned at = s * (S::stage_bytes >> 4);
          half_issue<false, 3, LAYOUT, low>(st.tmem + acc * 64, p_desc + at, q_desc + at, idesc, chunks - k * 4, !fresh);
          tcgen05_commit(st.empty + 8 * s);
          if (taken) {
            tcgen05_commit(st.acc_full + 8 * acc);
            ++st.t;
          }
        }
      });
    }
    __syncwarp();
  } else if (st.warp >= 4) {
    const unsigned quarter = st.warp & 3u, odd = st.warp >= 8;
    epilogue.box.phase = st.phase;
    each_tile([&](unsigned p0, unsigned q0) {
      const unsigned row0 = p0 + quarter * 32, column = q0 + odd * 32;
      const HalfPlace at = {st.matrix, 0, p0, q0, p0 / 128 * tiles_q + q0 / 64, 0, symmetric ? 128u : 1u << 30};      // no tile lies wholly above the diagonal: nothing is mirrored
      epilogue.begin(args, at, row0, odd);
      const bool inside = row0 < P && column < Q;
      if (inside) epilogue.ahead(args, column);
      float sum[32];
#pragma unroll
      for (unsigned q = 0; q < 32; ++q) sum[q] = 0.0f;
#pragma unroll 1
      for (unsigned k = 0; k < stages; k += kChunk, ++st.t) {
        const unsigned acc = st.t % S::accs;
        st.ok = __all_sync(0xFFFFFFFFu, mbarrier_wait(st.acc_full + 8 * acc, (st.t / S::accs) & 1u, 4 * kHalfPolls));
        if (!st.ok) break;
        tcgen05_fence_after();
        unsigned v[32];
        tmem_read32(st.tmem + acc * 64 + (quarter << 21) + odd * 32, v);
        tcgen05_fence_before();
        __syncwarp();
        if (st.lane == 0) mbarrier_arrive_cluster(st.acc_free + 8 * acc);
#pragma unroll
        for (unsigned q = 0; q < 32; ++q) sum[q] += __uint_as_float(v[q]);
      }
      if (st.ok && inside) epilogue.unit(args, column, min(32u, Q - column), sum);
      __syncwarp();
      if (st.ok) epilogue.end(args, at, st.warp - 4);
      __syncwarp();
    });
  }
  if (st.warp >= 4) {
    epilogue.box.finish();                      // what has been sent is there
    st.ok = st.ok && epilogue.box.fine;
    st.phase = epilogue.box.phase;
  }
}

template <bool TALL, int TO, typename T>
__global__ void __launch_bounds__(kHalfThreads, 1)
orthogonal_cluster_kernel(const __grid_constant__ ClusterArgs<TO, T> a) {
  using S = ClusterShape;
  extern __shared__ __align__(1024) unsigned char cluster_smem[];
  uint64_t* bars = reinterpret_cast<uint64_t*>(cluster_smem + S::stages * S::stage_bytes + S::out_bytes);
  unsigned &tmem_base = *reinterpret_cast<unsigned*>(bars + 2 * S::stages + 1 + 16 + 2 * S::accs), &failed = *(&tmem_base + 1);
  ClusterState st;
  st.stage0 = smem_u32(cluster_smem);
  st.full = smem_u32(bars);
  st.empty = st.full + 8 * S::stages;
  st.acc_full = st.empty + 8 * S::stages;
  st.acc_free = st.acc_full + 8 * S::accs;
  const unsigned box_full = st.acc_free + 8 * S::accs;
  st.warp = threadIdx.x >> 5;
  st.lane = threadIdx.x & 31u;
  st.rank = cluster_rank();
  st.size = cluster_size();
  st.matrix = blockIdx.x / st.size;
  st.starve = a.starve;
  st.n = st.t = st.phase = 0;
  st.ok = true;
  if (threadIdx.x == 0) {
    prefetch_tensor_map(&a.x[0][0]);
    prefetch_tensor_map(&a.x[0][1]);
    for (unsigned s = 0; s < S::stages; ++s) {
      mbarrier_init(st.full + 8 * s, 1);
      mbarrier_init(st.empty + 8 * s, 1);
    }
    for (unsigned b = 0; b < S::accs; ++b) {
      mbarrier_init(st.acc_full + 8 * b, 1);
      mbarrier_init(st.acc_free + 8 * b, 8);
    }
    for (unsigned b = 0; b < 16; ++b) mbarrier_init(box_full + 8 * b, 1);
    mbarrier_init_fence();
    failed = 0;
  }
  pdl_launch_dependents();
  pdl_wait();                                   // before tensor memory is taken: its last holder has finished
  if (st.warp == 1) tmem_alloc(smem_u32(&tmem_base), S::columns);
  tcgen05_fence_before();
  __syncthreads();
  tcgen05_fence_after();
  st.tmem = tmem_base;

  const unsigned side = TALL ? a.cols : a.rows, other = TALL ? a.rows : a.cols, w = st.warp >= 4 ? st.warp - 4 : 0;
  // half of the tiles of a square, mirrored, where that saves a round
  const unsigned squares = (side + 127) / 128 * ((side + 63) / 64);
  const bool symmetric = squares > st.size;
  const Box box(st.stage0 + S::stages * S::stage_bytes + w * S::box_bytes, box_full + 16 * w, st.lane);
  GramEpilogue<true> gram(a.gram[0], box);
  PolynomialEpilogue<true, 2> polynomial(a.polynomial, box);
  UpdateEpilogue<kNextStep, float, 2> next(a.next[0], box);
  UpdateEpilogue<TO, T, 2> last(a.last, box);
  // All CTAs of the cluster have left a product behind.  A CTA that gave up keeps step and does nothing more.
  auto between = [&]() {
    if (!st.ok) atomicExch(&failed, 1u);
    proxy_fence();
    __syncwarp();
    cluster_sync();
    proxy_fence();
    st.ok = *(volatile unsigned*)&failed == 0;
  };
  for (unsigned k = 0; k < a.steps; ++k) {
    const CUtensorMap* x = a.x[k & 1u];
    gram.seen = ~0u;                            // another step, another d
    cluster_product<TALL ? kBothByRows : kBothByK>(st, symmetric, x, x, side, side, other, gram, a.gram[k > 0]);
    between();
    cluster_product<kBothByK>(st, symmetric, a.e, a.e, side, side, side, polynomial, a.polynomial);
    between();
    if (k + 1 < a.steps) {
      if (TALL) cluster_product<kBothByK>(st, false, x, a.m, a.rows, a.cols, side, next, a.next[k & 1u]);
      else cluster_product<kQByRows>(st, false, a.m, x, a.rows, a.cols, side, next, a.next[k & 1u]);
    } else {
      if (TALL) cluster_product<kBothByK>(st, false, x, a.m, a.rows, a.cols, side, last, a.last);
      else cluster_product<kQByRows>(st, false, a.m, x, a.rows, a.cols, side, last, a.last);
    }
    between();
  }
  // the last stages' commits have to arrive, and where a wait ran out, the copies that were asked for
  if (st.warp == 0 && st.n > 0)
    for (unsigned m = st.n > S::stages ? st.n - S::stages : 0; m < st.n; ++m) {
      const bool there = mbarrier_wait(st.empty + 8 * (m % S::stages), (m / S::stages) & 1u, st.ok ? kHalfPolls : 1000u);
      if (!there) (void)mbarrier_wait(st.full + 8 * (m % S::stages), (m / S::stages) & 1u, st.ok ? kHalfPolls : 1000u);
    }
  __syncthreads();
  if (threadIdx.x == 0 && failed) atomicOr(a.status, 1u);
  if (st.warp == 1) {
    tcgen05_fence_after();
    tmem_free(st.tmem, S::columns);
  }
}

// ---------------------------------------------------------------------------------------------------------------------
// Host side.

constexpr size_t kMostSide = SSGD_ORTHOGONAL_MAX_SIDE;
inline size_t round_up(size_t n, size_t k) { return (n + k - 1) / k * k; }

struct Layout {
  size_t side, ldx, lds, x_elements, e_elements;        // of one matrix
  unsigned norm_parts, square_parts;                    // square_parts: most that any form of the update leaves
  size_t partial, d, squares, x, e, bytes;              // offsets; x: four matrices' parts, e: four
};
inline bool layout_of(size_t n, size_t rows, size_t cols, Layout* l) {
  if (n < 1 || n > 65535 || rows < 1 || cols < 1 || rows > kMostSide || cols > kMostSide) return false;
  l->side = rows < cols ? rows : cols;
  l->ldx = round_up(cols, 64);
  l->lds = round_up(l->side, 64);
  l->x_elements = rows * l->ldx;
  l->e_elements = l->side * l->lds;
  const size_t work = rows * ((cols + 7) / 8);
  l->norm_parts = (unsigned)((work + 4 * kNormThreads - 1) / (4 * kNormThreads));
  const unsigned most = n >= 16 ? 96 : 1184;            // CTAs of one matrix
  if (l->norm_parts > most) l->norm_parts = most;
  l->square_parts = (unsigned)(16 * ((rows + 127) / 128) * ((cols + 63) / 64));
  size_t at = 0;
  l->partial = at; at += round_up(n * l->norm_parts * 8, 128);
  l->d = at; at += round_up(n * 4, 128);
  l->squares = at; at += round_up(n * l->square_parts * 4, 128);
  l->x = at; at += 4 * round_up(n * l->x_elements * 2, 128);
  l->e = at; at += 4 * round_up(n * l->e_elements * 2, 128);
  l->bytes = at;
  return true;
}

struct Problem {
  Source source;
  int source_type;
  bool momentum;
  size_t n, rows, cols;
  Polynomial f;
  unsigned steps;
  int terms;
  void* out;                    // of out_type, or with a momentum the parameters
  int out_type;
  size_t ldo, out_stride;
  float delta;
  char* ws;
  unsigned* status;
  unsigned starve;
};

template <int KIND, typename T>
ssgd_status launch_source(const Problem& p, const Layout& l, const Whole& x, cudaStream_t s) {
  double* partial = reinterpret_cast<double*>(p.ws + l.partial);
  const dim3 grid(l.norm_parts, (unsigned)p.n);
  launch_kernel(orthogonal_norm_kernel<KIND, T>, grid, dim3(kNormThreads), 0, s, true, p.source, partial);
  launch_kernel(orthogonal_split_kernel<KIND, T>, grid, dim3(kNormThreads), 0, s, true, p.source, static_cast<const double*>(partial), l.norm_parts, x);
  return launch_status();
}
template <int KIND>
ssgd_status launch_source_typed(const Problem& p, const Layout& l, const Whole& x, cudaStream_t s) {
  switch (p.source_type) {
    case SSGD_F32: return launch_source<KIND, float>(p, l, x, s);
    case SSGD_BF16: return launch_source<KIND, __nv_bfloat16>(p, l, x, s);
    default: return launch_source<KIND, __half>(p, l, x, s);
  }
}

struct Buffers {
  Whole x[2], e, m;
  Parts x_parts[2], e_parts, m_parts;
  float *d, *squares;
};

// One product: tiles of 256 columns and three terms leave an epilogue one box.
template <template <unsigned> class Epilogue, int TERMS, int LAYOUT, typename Args>
ssgd_status launch_boxed(const HalfProduct& h, const Args& args, const HalfForm& form, int sms, cudaStream_t s) {
  constexpr int chunk = TERMS == 3 ? kChunk : 0;
  if (form.nt == 256) {
    using Wide = Epilogue<TERMS == 3 ? 1 : 2>;
    return launch_half_form<Wide, true, 256, TERMS, 4 * chunk, LAYOUT, false>(h, args, 1, sms, s);
  }
  using Other = Epilogue<2>;
  return launch_narrow<Other, TERMS, chunk, LAYOUT>(h, args, form, 1, sms, s);
}
template <bool LOW>
struct GramOf { template <unsigned> using Epilogue = GramEpilogue<LOW>; };
template <bool LOW>
struct PolynomialOf { template <unsigned BOXES> using Epilogue = PolynomialEpilogue<LOW, BOXES>; };
template <int TO, typename T>
struct UpdateOf { template <unsigned BOXES> using Epilogue = UpdateEpilogue<TO, T, BOXES>; };

template <int TO, typename T, int TERMS>
ssgd_status launch_update(const Problem& p, const Layout& l, const Buffers& b, int now, unsigned* count, int sms, cudaStream_t s) {
  const Whole& x = b.x[now];
  const HalfOperand whole = {x.high, x.low, x.ld, x.stride, false}, square = {b.m.high, b.m.low, b.m.ld, b.m.stride, false};
  HalfProduct h = {};
  h.P = p.rows; h.Q = p.cols; h.K = l.side; h.batch = p.n;
  h.status = p.status;
  h.starve = p.starve;
  if (p.rows <= p.cols) {                       // M X: X's columns are Q's rows
    h.p = square;
    h.q = whole;
    h.q.by_rows = true;
  } else {                                      // X M
    h.p = whole;
    h.q = square;
  }
  const HalfForm form = half_form(h, TERMS, 1, sms);
  const unsigned slots = form.pairs ? 16 : 8;                  // epilogue warps of a tile
  *count = slots * (unsigned)half_tiles(h, form.pairs ? 256 : 128, form.nt);
  UpdateArgs<T> a = {};
  a.x = b.x_parts[now]; a.next = b.x_parts[1 - now]; a.d = b.d; a.squares = b.squares;
  a.out = static_cast<T*>(p.out); a.ldo = p.ldo; a.out_stride = p.out_stride;
  a.f = p.f; a.delta = p.delta; a.rows = (unsigned)p.rows; a.count = *count; a.slots = slots;
  return h.q.by_rows ? launch_boxed<UpdateOf<TO, T>::template Epilogue, TERMS, kQByRows>(h, a, form, sms, s)
                     : launch_boxed<UpdateOf<TO, T>::template Epilogue, TERMS, kBothByK>(h, a, form, sms, s);
}

template <int TERMS>
ssgd_status newton_schulz(const Problem& p, const Layout& l, const Buffers& b, int sms, cudaStream_t s) {
  constexpr bool kLow = TERMS == 3;
  unsigned count = 0;
  int now = 0;
  for (unsigned k = 0; k < p.steps; ++k) {
    const Whole& x = b.x[now];
    HalfProduct h = {};
    h.p = {x.high, x.low, x.ld, x.stride, p.rows > p.cols};
    h.q = h.p;
    h.P = h.Q = l.side;
    h.K = p.rows > p.cols ? p.rows : p.cols;
    h.batch = p.n;
    h.symmetric = true;
    h.status = p.status;
    h.starve = p.starve;
    const typename GramEpilogue<kLow>::Args gram = {b.e_parts, k ? b.squares : nullptr, b.d, count, (unsigned)l.side};
    const HalfForm form = half_form(h, TERMS, 1, sms);
    ssgd_status st = h.p.by_rows ? launch_boxed<GramOf<kLow>::template Epilogue, TERMS, kBothByRows>(h, gram, form, sms, s)
                                 : launch_boxed<GramOf<kLow>::template Epilogue, TERMS, kBothByK>(h, gram, form, sms, s);
    if (st != SSGD_OK) return st;
    h.p = {b.e.high, b.e.low, b.e.ld, b.e.stride, false};
    h.q = h.p;
    h.K = l.side;
    const PolynomialArgs polynomial = {b.e_parts, b.m_parts, b.d, p.f};
    st = launch_boxed<PolynomialOf<kLow>::template Epilogue, TERMS, kBothByK>(h, polynomial, half_form(h, TERMS, 1, sms), sms, s);
    if (st != SSGD_OK) return st;
    if (k + 1 < p.steps) st = launch_update<kNextStep, float, TERMS>(p, l, b, now, &count, sms, s);
    else if (p.momentum) st = launch_update<kParameters, float, TERMS>(p, l, b, now, &count, sms, s);
    else if (p.out_type == SSGD_F32) st = launch_update<kOut, float, TERMS>(p, l, b, now, &count, sms, s);
    else if (p.out_type == SSGD_BF16) st = launch_update<kOut, __nv_bfloat16, TERMS>(p, l, b, now, &count, sms, s);
    else st = launch_update<kOut, __half, TERMS>(p, l, b, now, &count, sms, s);
    if (st != SSGD_OK) return st;
    now = 1 - now;
  }
  return SSGD_OK;
}

inline bool parts_of(Parts* parts, const Whole& w, size_t rows, size_t cols, size_t n) {
  return box_map(&parts->high, w.high, false, rows, cols, w.ld, n, w.stride) && box_map(&parts->low, w.low, false, rows, cols, w.ld, n, w.stride);
}

// A cluster for each matrix, where that is faster; the clocks of one step either way.  By launches: each product its own, and 5000 for the gap
// between two.  By a cluster: tiles of 128 x 64 in rounds, 1000 a stage and 4500 beside (a trip through L2, the epilogue, the barrier); on 148
// SMs clusters of 16 are counted as 6 at one time, of 8 as 12, of 4 as 24, of 2 as 48, on others in proportion.  (Of 4 and 2 there is room for 32 and 72:
// five steps of 24, 32, 36 and 64 matrices of 200 x 128 take 73, 74, 135 us by clusters and 110 by launches.)  0: launches.
inline unsigned cluster_ctas(const Problem& p, const Layout& l, int sms) {
  const size_t s = l.side, other = p.rows > p.cols ? p.rows : p.cols;
  HalfProduct h = {};
  h.P = h.Q = s;
  h.K = other;
  h.batch = p.n;
  h.symmetric = true;
  const unsigned long long square_tiles = half_tiles(h, 128, 64);
  unsigned long long launches = 3 * 5000ull, least = 0;
  (void)half_form(h, p.terms, 1, sms, &least);
  launches += least;
  h.K = s;
  (void)half_form(h, p.terms, 1, sms, &least);
  launches += least;
  h.P = p.rows; h.Q = p.cols; h.symmetric = false;
  (void)half_form(h, p.terms, 1, sms, &least);
  launches += least;
  const unsigned long long tiles = half_tiles(h, 128, 64), most = tiles > square_tiles ? tiles : square_tiles;
  const unsigned ctas = most <= 2 ? 2 : most <= 4 ? 4 : most <= 8 ? 8 : 16, counted = (ctas == 16 ? 6 : 96 / ctas) * (unsigned)sms / 148, at_once = counted ? counted : 1;
  const unsigned long long square_rounds = (square_tiles + ctas - 1) / ctas, rounds = (tiles + ctas - 1) / ctas;
  const unsigned long long stages = (other + 63) / 64, stages_s = (s + 63) / 64;
  const unsigned long long cluster = (square_rounds * (stages + stages_s) + rounds * stages_s) * 1000 + 3 * 4500;
  return cluster * ((p.n + at_once - 1) / at_once) < launches ? ctas : 0;
}

template <bool TALL, int TO, typename T>
ssgd_status launch_cluster(const Problem& p, const Layout& l, const Buffers& b, unsigned ctas, cudaStream_t s) {
  using S = ClusterShape;
  ClusterArgs<TO, T> a = {};
  auto operand = [&](CUtensorMap* maps, const Whole& w, size_t rows, size_t cols) {
    const HalfOperand o = {w.high, w.low, w.ld, w.stride, false};
    return half_map(&maps[0], w.high, false, o, rows, cols, p.n, 64) && half_map(&maps[1], w.low, false, o, rows, cols, p.n, 64);
  };
  if (!operand(a.x[0], b.x[0], p.rows, p.cols) || !operand(a.x[1], b.x[1], p.rows, p.cols) || !operand(a.e, b.e, l.side, l.side) ||
      !operand(a.m, b.m, l.side, l.side))
    return SSGD_ERR_CUDA;
  const unsigned count = 8 * (unsigned)(((p.rows + 127) / 128) * ((p.cols + 63) / 64));
  a.gram[0] = {b.e_parts, nullptr, b.d, count, (unsigned)l.side};
  a.gram[1] = {b.e_parts, b.squares, b.d, count, (unsigned)l.side};
  a.polynomial = {b.e_parts, b.m_parts, b.d, p.f};
  for (int i = 0; i < 2; ++i) {
    a.next[i].x = b.x_parts[i];
    a.next[i].next = b.x_parts[1 - i];
    a.next[i].d = b.d; a.next[i].squares = b.squares; a.next[i].f = p.f;
    a.next[i].rows = (unsigned)p.rows; a.next[i].count = count; a.next[i].slots = 8;
  }
  a.last.x = b.x_parts[(p.steps - 1) & 1u]; a.last.d = b.d; a.last.f = p.f;
  a.last.out = static_cast<T*>(p.out); a.last.ldo = p.ldo; a.last.out_stride = p.out_stride;
  a.last.delta = p.delta; a.last.rows = (unsigned)p.rows;
  a.rows = (unsigned)p.rows; a.cols = (unsigned)p.cols; a.steps = p.steps; a.starve = p.starve; a.status = p.status;
  auto kernel = orthogonal_cluster_kernel<TALL, TO, T>;
  static unsigned long long seen = 0, seen_wide = 0;
  if (!allow_smem(reinterpret_cast<const void*>(kernel), S::smem, &seen)) return SSGD_ERR_CUDA;
  cudaLaunchConfig_t cfg = {};
  cfg.blockDim = dim3(kHalfThreads);
  cfg.dynamicSmemBytes = S::smem;
  cfg.stream = s;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = ctas;
  attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 2;
  cfg.gridDim = dim3((unsigned)p.n * ctas);
  if (ctas > 8 && !allow_wide_clusters(reinterpret_cast<const void*>(kernel), cfg, &seen_wide)) {
    attr[1].val.clusterDim.x = ctas = 8;
    cfg.gridDim = dim3((unsigned)p.n * ctas);
  }
  (void)cudaLaunchKernelEx(&cfg, kernel, a);
  return launch_status();
}
template <int TO, typename T>
ssgd_status launch_cluster_any(const Problem& p, const Layout& l, const Buffers& b, unsigned ctas, cudaStream_t s) {
  return p.rows > p.cols ? launch_cluster<true, TO, T>(p, l, b, ctas, s) : launch_cluster<false, TO, T>(p, l, b, ctas, s);
}
ssgd_status by_cluster(const Problem& p, const Layout& l, const Buffers& b, unsigned ctas, cudaStream_t s) {
  if (p.momentum) return launch_cluster_any<kParameters, float>(p, l, b, ctas, s);
  switch (p.out_type) {
    case SSGD_F32: return launch_cluster_any<kOut, float>(p, l, b, ctas, s);
    case SSGD_BF16: return launch_cluster_any<kOut, __nv_bfloat16>(p, l, b, ctas, s);
    default: return launch_cluster_any<kOut, __half>(p, l, b, ctas, s);
  }
}

inline bool eights_of(const void* p, size_t element, size_t ld, size_t stride, size_t n) {
  const size_t of = 16 / element;               // elements of 16 bytes
  return aligned16(p) && ld % of == 0 && (n == 1 || stride % of == 0);
}

// One batch of matrices: rows of stride ld, matrices of stride `stride`, in elements of `type`.
ssgd_status check_batch(const void* p, int type, size_t n, size_t rows, size_t cols, size_t ld, size_t stride) {
  const size_t e = dtype_bytes((unsigned)type);
  if (e == 0) return SSGD_ERR_ARG;
  if (!p) return SSGD_ERR_NULL;
  if (reinterpret_cast<uintptr_t>(p) % e != 0) return SSGD_ERR_ALIGN;
  if (ld < cols || ld >= (size_t)1 << 44 || stride >= (size_t)1 << 44) return SSGD_ERR_SIZE;
  return SSGD_OK;
}
// Matrices that are written may not share elements: they lie behind one another, or their rows in turn.
inline bool overlapping(size_t n, size_t rows, size_t cols, size_t ld, size_t stride) {
  return n > 1 && stride < (rows - 1) * ld + cols && (stride < cols || ld < (n - 1) * stride + cols);
}

ssgd_status check_problem(size_t n, size_t rows, size_t cols, const float* coefficients, unsigned steps, int products, const void* ws, const unsigned* status) {
  if (rows < 1 || cols < 1 || rows > kMostSide || cols > kMostSide || n > 65535 || steps < 1 || steps > 100) return SSGD_ERR_SIZE;
  if (products != 1 && products != 3) return SSGD_ERR_ARG;
  if (!coefficients || !ws || !status) return SSGD_ERR_NULL;
  for (int i = 0; i < 3; ++i)
    if (!isfinite(coefficients[i])) return SSGD_ERR_ARG;
  if (!aligned16(ws) || (reinterpret_cast<uintptr_t>(status) & 3u)) return SSGD_ERR_ALIGN;
  return SSGD_OK;
}

ssgd_status solve_small(const Problem& p, cudaStream_t s) {
  static unsigned long long seen = 0;
  if (!allow_smem(reinterpret_cast<const void*>(orthogonal_small_kernel), kSmallSmem, &seen)) return SSGD_ERR_CUDA;
  const SmallArgs a = {p.source, p.source_type, p.out_type, p.momentum, p.out, p.ldo, p.out_stride, p.f, p.delta, p.steps, p.starve, p.status};
  launch_kernel(orthogonal_small_kernel, dim3((unsigned)p.n), dim3(kSmallThreads), kSmallSmem, s, true, a);
  return launch_status();
}

ssgd_status solve(Problem p, const float* coefficients, cudaStream_t s) {
  p.f = {coefficients[0], coefficients[1], coefficients[2]};
  if (p.rows <= kSmallSide && p.cols <= kSmallSide) return solve_small(p, s);
  DeviceInfo info;
  if (!device_info(&info)) return SSGD_ERR_CUDA;
  Layout l;
  if (!layout_of(p.n, p.rows, p.cols, &l)) return SSGD_ERR_SIZE;
  Buffers b;
  char* x = p.ws + l.x;
  const size_t whole = round_up(p.n * l.x_elements * 2, 128), square = round_up(p.n * l.e_elements * 2, 128);
  auto half_at = [](char* at) { return reinterpret_cast<__half*>(at); };
  for (int i = 0; i < 2; ++i) b.x[i] = {half_at(x + (2 * i) * whole), half_at(x + (2 * i + 1) * whole), l.ldx, l.x_elements};
  char* e = p.ws + l.e;
  b.e = {half_at(e), half_at(e + square), l.lds, l.e_elements};
  b.m = {half_at(e + 2 * square), half_at(e + 3 * square), l.lds, l.e_elements};
  if (!parts_of(&b.x_parts[0], b.x[0], p.rows, p.cols, p.n) || !parts_of(&b.x_parts[1], b.x[1], p.rows, p.cols, p.n) ||
      !parts_of(&b.e_parts, b.e, l.side, l.side, p.n) || !parts_of(&b.m_parts, b.m, l.side, l.side, p.n))
    return SSGD_ERR_CUDA;
  b.d = reinterpret_cast<float*>(p.ws + l.d);
  b.squares = reinterpret_cast<float*>(p.ws + l.squares);
  const ssgd_status st = p.momentum ? launch_source_typed<kMomentum>(p, l, b.x[0], s) : launch_source_typed<kPlainSource>(p, l, b.x[0], s);
  if (st != SSGD_OK) return st;
  if (const unsigned ctas = cluster_ctas(p, l, info.sms)) return by_cluster(p, l, b, ctas, s);
  return p.terms == 3 ? newton_schulz<3>(p, l, b, info.sms, s) : newton_schulz<1>(p, l, b, info.sms, s);
}

ssgd_status checked_orthogonalise(const void* u, int u_type, size_t n, size_t rows, size_t cols, size_t ldu, size_t stride_u, const float* coefficients,
                                  unsigned steps, int products, void* out, int out_type, size_t ldo, size_t stride_o, void* ws, unsigned* status,
                                  unsigned starve, void* stream) {
  if (n == 0) return SSGD_OK;
  ssgd_status st = check_problem(n, rows, cols, coefficients, steps, products, ws, status);
  if (st == SSGD_OK) st = check_batch(u, u_type, n, rows, cols, ldu, stride_u);
  if (st == SSGD_OK) st = check_batch(out, out_type, n, rows, cols, ldo, stride_o);
  if (st != SSGD_OK) return st;
  if (overlapping(n, rows, cols, ldo, stride_o)) return SSGD_ERR_SIZE;
  Problem p = {};
  p.source.u = u; p.source.ldu = ldu; p.source.u_stride = stride_u;
  p.source.rows = (unsigned)rows; p.source.cols = (unsigned)cols;
  p.source.eights = eights_of(u, dtype_bytes((unsigned)u_type), ldu, stride_u, n);
  p.source_type = u_type;
  p.n = n; p.rows = rows; p.cols = cols; p.steps = steps; p.terms = products;
  p.out = out; p.out_type = out_type; p.ldo = ldo; p.out_stride = stride_o;
  p.ws = static_cast<char*>(ws); p.status = status; p.starve = starve;
  return solve(p, coefficients, static_cast<cudaStream_t>(stream));
}

}  // namespace

extern "C" {

size_t ssgd_orthogonal_ws_bytes(size_t n, size_t rows, size_t cols) {
  Layout l;
  return layout_of(n, rows, cols, &l) ? l.bytes : 0;
}

ssgd_status ssgd_orthogonalise(const void* u, int u_type, size_t n, size_t rows, size_t cols, size_t ldu, size_t stride_u, const float* coefficients,
                               unsigned steps, int products, void* out, int out_type, size_t ldo, size_t stride_o, void* ws, unsigned* status, void* stream) {
  return checked_orthogonalise(u, u_type, n, rows, cols, ldu, stride_u, coefficients, steps, products, out, out_type, ldo, stride_o, ws, status, 0, stream);
}

ssgd_status ssgd_orthogonal_wait_selftest(const void* u, int u_type, size_t rows, size_t cols, const float* coefficients, int products, void* out,
                                          int out_type, void* ws, unsigned* status, void* stream) {
  if (rows > 256 || cols > 256) return SSGD_ERR_SIZE;       // one step, three products: their waits run out once each
  return checked_orthogonalise(u, u_type, 1, rows, cols, cols, rows * cols, coefficients, 1, products, out, out_type, cols, rows * cols, ws, status, 16, stream);
}

ssgd_status ssgd_orthogonal_step(float* x, size_t ldx, size_t stride_x, const void* g, int g_type, size_t ldg, size_t stride_g, float* m, size_t ldm,
                                 size_t stride_m, size_t n, size_t rows, size_t cols, float beta, float delta, int nesterov, const float* coefficients,
                                 unsigned steps, int products, void* ws, unsigned* status, void* stream) {
  if (!beta_ok(beta) || !isfinite(delta)) return SSGD_ERR_ARG;
  if (n == 0) return SSGD_OK;
  ssgd_status st = check_problem(n, rows, cols, coefficients, steps, products, ws, status);
  if (st == SSGD_OK) st = check_batch(x, SSGD_F32, n, rows, cols, ldx, stride_x);
  if (st == SSGD_OK) st = check_batch(g, g_type, n, rows, cols, ldg, stride_g);
  if (st == SSGD_OK) st = check_batch(m, SSGD_F32, n, rows, cols, ldm, stride_m);
  if (st != SSGD_OK) return st;
  if (overlapping(n, rows, cols, ldx, stride_x) || overlapping(n, rows, cols, ldm, stride_m)) return SSGD_ERR_SIZE;
  Problem p = {};
  p.source.u = g; p.source.ldu = ldg; p.source.u_stride = stride_g;
  p.source.m = m; p.source.ldm = ldm; p.source.m_stride = stride_m;
  p.source.beta = beta; p.source.ahead = nesterov != 0;
  p.source.rows = (unsigned)rows; p.source.cols = (unsigned)cols;
  p.source.eights = eights_of(g, dtype_bytes((unsigned)g_type), ldg, stride_g, n) && eights_of(m, 4, ldm, stride_m, n);
  p.source_type = g_type;
  p.momentum = true;
  p.n = n; p.rows = rows; p.cols = cols; p.steps = steps; p.terms = products;
  p.out = x; p.out_type = SSGD_F32; p.ldo = ldx; p.out_stride = stride_x; p.delta = delta;
  p.ws = static_cast<char*>(ws); p.status = status;
  return solve(p, coefficients, static_cast<cudaStream_t>(stream));
}

ssgd_status ssgd_orthogonalise_block(const uint64_t* a) {
  if (!a) return SSGD_ERR_NULL;
  const float c[3] = {block_float(a[7]), block_float(a[8]), block_float(a[9])};
  return ssgd_orthogonalise(block_ptr<const void>(a[0]), (int)a[1], a[2], a[3], a[4], a[5], a[6], c, (unsigned)a[10], (int)a[11], block_ptr<void>(a[12]),
                            (int)a[13], a[14], a[15], block_ptr<void>(a[16]), block_ptr<unsigned>(a[17]), block_ptr<void>(a[18]));
}

ssgd_status ssgd_orthogonal_step_block(const uint64_t* a) {
  if (!a) return SSGD_ERR_NULL;
  const float c[3] = {block_float(a[16]), block_float(a[17]), block_float(a[18])};
  return ssgd_orthogonal_step(block_ptr<float>(a[0]), a[1], a[2], block_ptr<const void>(a[3]), (int)a[4], a[5], a[6], block_ptr<float>(a[7]), a[8], a[9], a[10],
                              a[11], a[12], block_float(a[13]), block_float(a[14]), (int)a[15], c, (unsigned)a[19], (int)a[20], block_ptr<void>(a[21]),
                              block_ptr<unsigned>(a[22]), block_ptr<void>(a[23]));
}

}  // extern "C"
