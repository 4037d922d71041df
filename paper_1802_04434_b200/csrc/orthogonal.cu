// Orthogonalised updates: a matrix U with its singular values brought near one by Newton-Schulz products (what the Muon optimiser
// does with its momentum), and the whole momentum step with it.  See include/signsgd.h for the contract.
//
//   X = U / |U|_F, then `steps` times  X <- a X + (b A + c A^2) X,  A = X X^T       (rows <= columns; else from the right)
//
// Three products a step, on the tensor cores, A and A^2 by the tiles on and above their diagonals alone.  An fp16 operand has
// eleven bits, and what a step loses, the next ones multiply by up to a (a direction whose singular value is still small grows
// by that), so the arithmetic is arranged to lose little:
//   - with d = |X|_F^2 / s (s the shorter side), A = d I + E, and the step is  X <- (a + b d + c d^2) X + ((b + 2 c d) E + c E^2) X:  the
//     part along X is done in fp32, and what goes through fp16 shrinks as X approaches its goal (A near I, E small).  For 16-bit
//     results: error of X relative 4e-4 .. 1e-3, without this 2e-3 .. 3e-3; the rounding to bf16 alone is 1.7e-3
//   - X is kept as the sum of two fp16 matrices, so that (a + ..) X loses nothing
//   - TERMS = 3: products take both parts of each operand (22 bits; error 2e-7 .. 4e-6, an fp32 product's 1e-6 .. 1e-5); TERMS = 1:
//     the high parts alone
// All matrices are stored times 2^13: elements are at most 1.2 in size, and the smallest that count stay normal numbers of fp16.

#include "half_product.cuh"

namespace {

constexpr float kScale = 8192.0f, kUnscale = 1.0f / 8192.0f;      // of X, E and M as they are stored

struct Polynomial { float a, b, c; };
struct Step { float q, p, c; };                                    // X' = q X + (p E + c E^2) X
__device__ __forceinline__ Step step_of(const Polynomial& f, float d) {
  return {f.a + d * (f.b + d * f.c), f.b + 2.0f * f.c * d, f.c};
}

// What a value is stored as.
__device__ __forceinline__ void split_half(float v, __half* high, __half* low) {
  *high = __float2half_rn(v);
  *low = __float2half_rn(v - __half2float(*high));
}

// Eight neighbours of a row as high and low part.  The matrices' rows are padded to whole 64 columns, so that nobody has to ask
// where they end.
template <bool LOW>
__device__ __forceinline__ void store_split8(__half* high, __half* low, size_t at, const float* v) {
  float h[8];
#pragma unroll
  for (unsigned q = 0; q < 8; ++q) h[q] = __half2float(__float2half_rn(v[q]));
  store8(high + at, h);
  if constexpr (LOW) {
#pragma unroll
    for (unsigned q = 0; q < 8; ++q) h[q] = v[q] - h[q];
    store8(low + at, h);
  }
}
template <bool LOW>
__device__ __forceinline__ void load_split8(const __half* high, const __half* low, size_t at, float (&v)[8]) {
  load8(high + at, v);
  if constexpr (LOW) {
    float w[8];
    load8(low + at, w);
#pragma unroll
    for (unsigned q = 0; q < 8; ++q) v[q] += w[q];
  }
}

struct Square {                   // a batch of symmetric matrices, high and low part
  __half *high, *low;
  size_t ld, stride;
  unsigned side;
};

// A thread's 32 columns of a row of a symmetric matrix: there, and, from tiles wholly above the diagonal, mirrored (lanes side by
// side).  Tiles on the diagonal hold both halves themselves.
template <bool LOW>
__device__ __forceinline__ void store_symmetric(const Square& s, size_t matrix, unsigned row, unsigned column, unsigned left, bool mirrored, const float (&v)[32]) {
#pragma unroll
  for (unsigned c = 0; c < 32; c += 8) store_split8<LOW>(s.high, s.low, matrix + (size_t)row * s.ld + column + c, v + c);
  if (mirrored) {
#pragma unroll
    for (unsigned q = 0; q < 32; ++q) {
      if (q < left) {
        __half high, low;
        split_half(v[q], &high, &low);
        s.high[matrix + (size_t)(column + q) * s.ld + row] = high;
        if (LOW) s.low[matrix + (size_t)(column + q) * s.ld + row] = low;
      }
    }
  }
}

// E = X X^T - d I.  d comes from the sums of squares that the last step left, added in a fixed order by each warp; the first tile
// of each matrix leaves it for the other two products.
template <bool LOW>
struct GramEpilogue {
  struct Args {
    Square e;
    const float* squares;       // [matrix][count], or null: |X| is 1
    float* d;                   // [matrix]
    unsigned count;
  };
  float d;
  unsigned row, seen;
  size_t matrix;
  bool mirrored, inside;
  __device__ __forceinline__ GramEpilogue(const Args&, unsigned char*) { seen = ~0u; }
  __device__ __forceinline__ void begin(const Args& a, const HalfPlace& at, unsigned row0, unsigned lane, unsigned) {
    row = row0 + lane;
    inside = row < a.e.side;
    mirrored = at.q0 >= at.p0 + at.rows;
    matrix = at.matrix * a.e.stride;
    if (at.matrix != seen) {
      seen = at.matrix;
      float sum = 1.0f;
      if (a.squares) {
        sum = 0.0f;
        for (unsigned i = lane; i < a.count; i += 32) sum += a.squares[(size_t)at.matrix * a.count + i];
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xFFFFFFFFu, sum, o);
      }
      d = sum / (float)a.e.side;
    }
    if (at.tile == 0 && row == 0) a.d[at.matrix] = d;      // two warps: the same value
  }
  __device__ __forceinline__ void unit(const Args& a, unsigned column, unsigned left, float (&v)[32]) {
    if (!inside) return;
#pragma unroll
    for (unsigned q = 0; q < 32; ++q) v[q] *= kUnscale;
    if (row - column < 32u) {
#pragma unroll
      for (unsigned q = 0; q < 32; ++q)
        v[q] = row - column == q ? v[q] - d * kScale : v[q];
    }
    store_symmetric<LOW>(a.e, matrix, row, column, left, mirrored, v);
  }
  __device__ __forceinline__ void end(const Args&, const HalfPlace&, unsigned) {}
  __device__ __forceinline__ void finish() {}
};

// M = p E + c E^2.
template <bool LOW>
struct PolynomialEpilogue {
  struct Args {
    Square e, m;
    const float* d;
    Polynomial f;
  };
  Step s;
  unsigned row;
  size_t matrix;
  bool mirrored, inside;
  __device__ __forceinline__ PolynomialEpilogue(const Args&, unsigned char*) {}
  __device__ __forceinline__ void begin(const Args& a, const HalfPlace& at, unsigned row0, unsigned lane, unsigned) {
    row = row0 + lane;
    inside = row < a.e.side;
    mirrored = at.q0 >= at.p0 + at.rows;
    matrix = at.matrix * a.e.stride;
    s = step_of(a.f, a.d[at.matrix]);
  }
  __device__ __forceinline__ void unit(const Args& a, unsigned column, unsigned left, float (&v)[32]) {
    if (!inside) return;
#pragma unroll
    for (unsigned c = 0; c < 32; c += 8) {
      float e[8];
      load_split8<LOW>(a.e.high, a.e.low, matrix + (size_t)row * a.e.ld + column + c, e);
#pragma unroll
      for (unsigned q = 0; q < 8; ++q) v[c + q] = fmaf(s.c, v[c + q] * kUnscale, s.p * e[q]);
    }
    store_symmetric<LOW>(a.m, matrix, row, column, left, mirrored, v);
  }
  __device__ __forceinline__ void end(const Args&, const HalfPlace&, unsigned) {}
  __device__ __forceinline__ void finish() {}
};

struct Whole {                    // a batch of matrices X, high and low part
  __half *high, *low;
  size_t ld, stride;
};

// X' = q X + M X: kept for the next step, with its sum of squares; or, behind the last, written out as T; or x <- x - delta X'.
enum UpdateTo { kNextStep, kOut, kParameters };
template <int TO, typename T>
struct UpdateEpilogue {
  struct Args {
    Whole x, next;
    const float* d;
    float* squares;             // [matrix][count]
    T* out;
    size_t ldo, out_stride;
    Polynomial f;
    float delta;
    unsigned rows, count, slots;        // sums of squares of a matrix, and of a tile
  };
  float q, sum;
  unsigned row;
  bool inside;
  size_t at_x;
  T* out;
  __device__ __forceinline__ UpdateEpilogue(const Args&, unsigned char*) {}
  __device__ __forceinline__ void begin(const Args& a, const HalfPlace& at, unsigned row0, unsigned lane, unsigned) {
    row = row0 + lane;
    inside = row < a.rows;
    at_x = at.matrix * a.x.stride + (size_t)row * a.x.ld;
    if (TO != kNextStep && inside) out = a.out + at.matrix * a.out_stride + (size_t)row * a.ldo;
    q = step_of(a.f, a.d[at.matrix]).q;
    sum = 0.0f;
  }
  __device__ __forceinline__ void unit(const Args& a, unsigned column, unsigned left, float (&v)[32]) {
    if (!inside) return;
    const bool wide = TO != kNextStep && left >= 32 && (reinterpret_cast<uintptr_t>(out + column) & 15u) == 0;
#pragma unroll
    for (unsigned c = 0; c < 32; c += 8) {
      float x[8];
      load_split8<true>(a.x.high, a.x.low, at_x + column + c, x);
#pragma unroll
      for (unsigned i = 0; i < 8; ++i) v[c + i] = fmaf(q, x[i], v[c + i] * kUnscale);
      if constexpr (TO == kNextStep) {
#pragma unroll
        for (unsigned i = 0; i < 8; ++i) sum = c + i < left ? fmaf(v[c + i], v[c + i], sum) : sum;
        store_split8<true>(a.next.high, a.next.low, at_x + column + c, v + c);
      } else if constexpr (TO == kOut) {
#pragma unroll
        for (unsigned i = 0; i < 8; ++i) v[c + i] *= kUnscale;
        if (wide) {
          store8(out + column + c, v + c);
        } else {
#pragma unroll
          for (unsigned i = 0; i < 8; ++i)
            if (c + i < left) out[column + c + i] = from_float<T>(v[c + i]);
        }
      } else {
        const float step = a.delta * kUnscale;
        if (wide) {
          load8(out + column + c, x);
#pragma unroll
          for (unsigned i = 0; i < 8; ++i) x[i] = fmaf(-step, v[c + i], x[i]);
          store8(out + column + c, x);
        } else {
#pragma unroll
          for (unsigned i = 0; i < 8; ++i)
            if (c + i < left) out[column + c + i] = fmaf(-step, v[c + i], out[column + c + i]);
        }
      }
    }
  }
  __device__ __forceinline__ void end(const Args& a, const HalfPlace& at, unsigned warp) {
    if constexpr (TO == kNextStep) {
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xFFFFFFFFu, sum, o);
      if ((threadIdx.x & 31u) == 0) a.squares[(size_t)at.matrix * a.count + at.tile * a.slots + warp] = sum * (kUnscale * kUnscale);
    }
  }
  __device__ __forceinline__ void finish() {}
};

// ---------------------------------------------------------------------------------------------------------------------
// Before the products: the norm, then X's two parts.  A momentum step makes its U on the way, in both passes the same:
//   m <- fma(beta, m, fl((1 - beta) g)),  u = m, or looking ahead fma(beta, m, fl((1 - beta) g))

struct Source {
  const void* u;                // the matrix itself; with a momentum the gradient
  float* m;
  size_t ldu, u_stride, ldm, m_stride;
  float beta;
  unsigned rows, cols;
  bool ahead, fours;            // fours: every row of u and m starts at a multiple of four elements
};
enum { kPlainSource, kMomentum };

template <typename T>
__device__ __forceinline__ void source_load(const T* p, unsigned left, bool fours, float (&v)[4]) {
  if (fours && left >= 4) {
    const float4 q = load4(p);
    v[0] = q.x; v[1] = q.y; v[2] = q.z; v[3] = q.w;
  } else {
#pragma unroll
    for (unsigned i = 0; i < 4; ++i) v[i] = i < left ? to_float(p[i]) : 0.0f;
  }
}

// U at four columns of a row; FIRST: m is brought forward and written.
template <int KIND, bool FIRST, typename T>
__device__ __forceinline__ void source_values(const Source& s, size_t matrix, unsigned row, unsigned column, float (&u)[4]) {
  const unsigned left = s.cols - column;
  if constexpr (KIND == kPlainSource) {
    source_load(static_cast<const T*>(s.u) + matrix * s.u_stride + (size_t)row * s.ldu + column, left, s.fours, u);
  } else {
    float* mp = s.m + matrix * s.m_stride + (size_t)row * s.ldm + column;
    float m[4], g[4];
    source_load(mp, left, s.fours, m);
    if (FIRST || s.ahead) {
      source_load(static_cast<const T*>(s.u) + matrix * s.u_stride + (size_t)row * s.ldu + column, left, s.fours, g);
#pragma unroll
      for (unsigned i = 0; i < 4; ++i) g[i] = __fmul_rn(1.0f - s.beta, g[i]);
    }
    if (FIRST) {
#pragma unroll
      for (unsigned i = 0; i < 4; ++i) m[i] = __fmaf_rn(s.beta, m[i], g[i]);
      if (s.fours && left >= 4) {
        *reinterpret_cast<float4*>(mp) = make_float4(m[0], m[1], m[2], m[3]);
      } else {
#pragma unroll
        for (unsigned i = 0; i < 4; ++i)
          if (i < left) mp[i] = m[i];
      }
    }
#pragma unroll
    for (unsigned i = 0; i < 4; ++i) u[i] = s.ahead ? __fmaf_rn(s.beta, m[i], g[i]) : m[i];
  }
}

constexpr unsigned kNormThreads = 256;

template <int KIND, typename T>
__global__ void __launch_bounds__(kNormThreads)
orthogonal_norm_kernel(const Source s, double* __restrict__ partial) {
  __shared__ double part[kNormThreads / 32];
  pdl_launch_dependents();
  pdl_wait();
  const unsigned fours = (s.cols + 3) / 4, total = fours * s.rows;
  double sum = 0.0;
  for (unsigned i = blockIdx.x * kNormThreads + threadIdx.x; i < total; i += gridDim.x * kNormThreads) {
    float u[4];
    source_values<KIND, true, T>(s, blockIdx.y, i / fours, i % fours * 4, u);
#pragma unroll
    for (unsigned k = 0; k < 4; ++k)
      if (i % fours * 4 + k < s.cols) sum = fma((double)u[k], (double)u[k], sum);
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xFFFFFFFFu, sum, o);
  if ((threadIdx.x & 31u) == 0) part[threadIdx.x >> 5] = sum;
  __syncthreads();
  if (threadIdx.x == 0) {
    for (unsigned w = 1; w < kNormThreads / 32; ++w) sum += part[w];
    partial[(size_t)blockIdx.y * gridDim.x + blockIdx.x] = sum;
  }
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
  // 1 / |U| in two factors, a power of two that brings |U| to [1, 2) where that is an fp32 number, and the rest: the first
  // multiplication is exact, and neither leaves fp32's range.  A zero matrix stays zero, one that is not finite becomes NaN.
  const double norm = sqrt(norm2);
  const int e = norm > 0.0 && isfinite(norm) ? max(-126, min(126, -ilogb(norm))) : 0;
  const float first = __uint_as_float((unsigned)(127 + e) << 23);
  const float rest = norm > 0.0 ? (isfinite(norm) ? (float)((double)kScale / (norm * (double)first)) : __uint_as_float(0x7FC00000u)) : 0.0f;
  const unsigned fours = (s.cols + 3) / 4, total = fours * s.rows;
  for (unsigned i = blockIdx.x * kNormThreads + threadIdx.x; i < total; i += gridDim.x * kNormThreads) {
    const unsigned row = i / fours, column = i % fours * 4;
    float u[4];
    source_values<KIND, false, T>(s, blockIdx.y, row, column, u);
    float h[4], l[4];
#pragma unroll
    for (unsigned k = 0; k < 4; ++k) {
      const float v = u[k] * first * rest;
      h[k] = __half2float(__float2half_rn(v));
      l[k] = v - h[k];
    }
    const size_t at = blockIdx.y * x.stride + (size_t)row * x.ld + column;
    *reinterpret_cast<uint2*>(x.high + at) = make_uint2(pack2(__half(), h[0], h[1]), pack2(__half(), h[2], h[3]));
    *reinterpret_cast<uint2*>(x.low + at) = make_uint2(pack2(__half(), l[0], l[1]), pack2(__half(), l[2], l[3]));
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
  const size_t work = rows * ((cols + 3) / 4);
  l->norm_parts = (unsigned)((work + 8 * kNormThreads - 1) / (8 * kNormThreads));
  const unsigned most = n >= 16 ? 64 : 592;             // CTAs of one matrix
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

// Stages between two times that a sum of three terms is taken.
constexpr int kChunk = 2;

struct Buffers {
  Whole x[2];
  Square e, m;
  float *d, *squares;
};

template <int TO, typename T, int TERMS>
ssgd_status launch_update(const Problem& p, const Buffers& b, int now, unsigned* count, int sms, cudaStream_t s) {
  const Whole& x = b.x[now];
  const HalfOperand whole = {x.high, x.low, x.ld, x.stride, false}, square = {b.m.high, b.m.low, b.m.ld, b.m.stride, false};
  HalfProduct h = {};
  h.P = p.rows; h.Q = p.cols; h.K = b.m.side; h.batch = p.n;
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
  typename UpdateEpilogue<TO, T>::Args a = {};
  a.x = x; a.next = b.x[1 - now]; a.d = b.d; a.squares = b.squares;
  a.out = static_cast<T*>(p.out); a.ldo = p.ldo; a.out_stride = p.out_stride;
  a.f = p.f; a.delta = p.delta; a.rows = (unsigned)p.rows; a.count = *count; a.slots = slots;
  return launch_half<UpdateEpilogue<TO, T>, TERMS, TERMS == 3 ? kChunk : 0>(h, a, form, 1, sms, s);
}

template <int TERMS>
ssgd_status newton_schulz(const Problem& p, const Layout& l, const Buffers& b, int sms, cudaStream_t s) {
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
    const typename GramEpilogue<TERMS == 3>::Args gram = {b.e, k ? b.squares : nullptr, b.d, count};
    ssgd_status st = launch_half<GramEpilogue<TERMS == 3>, TERMS, TERMS == 3 ? kChunk : 0>(h, gram, half_form(h, TERMS, 1, sms), 1, sms, s);
    if (st != SSGD_OK) return st;
    h.p = {b.e.high, b.e.low, b.e.ld, b.e.stride, false};
    h.q = h.p;
    h.K = l.side;
    const typename PolynomialEpilogue<TERMS == 3>::Args polynomial = {b.e, b.m, b.d, p.f};
    st = launch_half<PolynomialEpilogue<TERMS == 3>, TERMS, TERMS == 3 ? kChunk : 0>(h, polynomial, half_form(h, TERMS, 1, sms), 1, sms, s);
    if (st != SSGD_OK) return st;
    if (k + 1 < p.steps) st = launch_update<kNextStep, float, TERMS>(p, b, now, &count, sms, s);
    else if (p.momentum) st = launch_update<kParameters, float, TERMS>(p, b, now, &count, sms, s);
    else if (p.out_type == SSGD_F32) st = launch_update<kOut, float, TERMS>(p, b, now, &count, sms, s);
    else if (p.out_type == SSGD_BF16) st = launch_update<kOut, __nv_bfloat16, TERMS>(p, b, now, &count, sms, s);
    else st = launch_update<kOut, __half, TERMS>(p, b, now, &count, sms, s);
    if (st != SSGD_OK) return st;
    now = 1 - now;
  }
  return SSGD_OK;
}

inline bool fours_of(const void* p, size_t element, size_t ld, size_t stride, size_t n) {
  return reinterpret_cast<uintptr_t>(p) % (4 * element) == 0 && ld % 4 == 0 && (n == 1 || stride % 4 == 0);
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
// Matrices that are written may not share elements.
inline bool overlapping(size_t n, size_t rows, size_t cols, size_t ld, size_t stride) { return n > 1 && stride < (rows - 1) * ld + cols; }

ssgd_status check_problem(size_t n, size_t rows, size_t cols, const float* coefficients, unsigned steps, int products, const void* ws, const unsigned* status) {
  if (rows < 1 || cols < 1 || rows > kMostSide || cols > kMostSide || n > 65535 || steps < 1 || steps > 100) return SSGD_ERR_SIZE;
  if (products != 1 && products != 3) return SSGD_ERR_ARG;
  if (!coefficients || !ws || !status) return SSGD_ERR_NULL;
  for (int i = 0; i < 3; ++i)
    if (!isfinite(coefficients[i])) return SSGD_ERR_ARG;
  if (!aligned16(ws) || (reinterpret_cast<uintptr_t>(status) & 3u)) return SSGD_ERR_ALIGN;
  return SSGD_OK;
}

ssgd_status solve(Problem p, const float* coefficients, cudaStream_t s) {
  DeviceInfo info;
  if (!device_info(&info)) return SSGD_ERR_CUDA;
  Layout l;
  if (!layout_of(p.n, p.rows, p.cols, &l)) return SSGD_ERR_SIZE;
  p.f = {coefficients[0], coefficients[1], coefficients[2]};
  Buffers b;
  char* x = p.ws + l.x;
  const size_t whole = round_up(p.n * l.x_elements * 2, 128), square = round_up(p.n * l.e_elements * 2, 128);
  auto half_at = [](char* at) { return reinterpret_cast<__half*>(at); };
  for (int i = 0; i < 2; ++i) b.x[i] = {half_at(x + (2 * i) * whole), half_at(x + (2 * i + 1) * whole), l.ldx, l.x_elements};
  char* e = p.ws + l.e;
  b.e = {half_at(e), half_at(e + square), l.lds, l.e_elements, (unsigned)l.side};
  b.m = {half_at(e + 2 * square), half_at(e + 3 * square), l.lds, l.e_elements, (unsigned)l.side};
  b.d = reinterpret_cast<float*>(p.ws + l.d);
  b.squares = reinterpret_cast<float*>(p.ws + l.squares);
  const ssgd_status st = p.momentum ? launch_source_typed<kMomentum>(p, l, b.x[0], s) : launch_source_typed<kPlainSource>(p, l, b.x[0], s);
  if (st != SSGD_OK) return st;
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
  p.source.fours = fours_of(u, dtype_bytes((unsigned)u_type), ldu, stride_u, n);
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
  p.source.fours = fours_of(g, dtype_bytes((unsigned)g_type), ldg, stride_g, n) && fours_of(m, 4, ldm, stride_m, n);
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
