// Norm and clipping of gradients that come as many tensors, into the flat rows that the step takes.
// See include/signsgd.h for the contract of each call.
//
// The host cuts every tensor into tiles of at most kTile elements and writes them into a table (caller-owned
// memory, copied to the device once); a CTA takes one tile, so tensors of any number and size are one launch
// and no CTA gets more than its share.  Tiles of a group (a worker) are consecutive:
//   pass 1  tensors_norm_kernel    partial[tile] = sum of squares (or largest magnitude) of the tile
//   pass 2  norms_finish_kernel    norm of each group from its partials, in a fixed order
//   pass 3  tensors_scale_kernel   dst = c * src with c = max_norm / norm where norm > max_norm, else 1
// No atomics: the same inputs give the same bits.  Squares are summed in fp64, where the product of two fp32 numbers is
// exact and can neither overflow nor vanish.

#include <string.h>

#include "host_common.h"
#include "dtypes.cuh"

namespace {

constexpr unsigned kTile = 8192;          // elements of a tile: 32 per thread

struct Tile {                             // one entry of the table
  const void* src;
  void* dst;
  uint32_t n;
  uint32_t group;
  uint32_t types;                         // source type | destination type << 4
  uint32_t unused;                        // keeps an entry at 32 bytes
};
static_assert(sizeof(Tile) == 32, "table entry");

// Table layout: first_tile[groups + 1] (64 bit, padded to a multiple of 32 bytes), then the tiles.
inline size_t table_head_bytes(size_t groups) { return ((groups + 1) * sizeof(uint64_t) + 31) / 32 * 32; }

constexpr int kNormTwo = 0, kNormMax = 1;

template <int KIND>
__device__ __forceinline__ void norm_fold(double& acc, float v) {
  if constexpr (KIND == kNormTwo) {
    const double t = (double)v;
    acc = fma(t, t, acc);
  }
}

// |v| as ordered bits: NaN sorts above infinity, so one maximum carries it through.
__device__ __forceinline__ unsigned magnitude_bits(float v) { return __float_as_uint(v) & 0x7FFFFFFFu; }

template <int KIND, typename T>
__device__ __forceinline__ void tile_norm(const T* __restrict__ src, unsigned n, double& acc, unsigned& top) {
  const bool aligned = (reinterpret_cast<uintptr_t>(src) & (4 * sizeof(T) - 1)) == 0;
  const unsigned body = aligned ? n & ~3u : 0u;
#pragma unroll 8
  for (unsigned i = threadIdx.x * 4; i < body; i += kThreads * 4) {
    const float4 q = load4(src + i);
    if constexpr (KIND == kNormTwo) {
      norm_fold<KIND>(acc, q.x); norm_fold<KIND>(acc, q.y); norm_fold<KIND>(acc, q.z); norm_fold<KIND>(acc, q.w);
    } else {
      top = max(max(top, max(magnitude_bits(q.x), magnitude_bits(q.y))), max(magnitude_bits(q.z), magnitude_bits(q.w)));
    }
  }
#pragma unroll 8
  for (unsigned i = body + threadIdx.x; i < n; i += kThreads) {
    const float v = to_float(src[i]);
    if constexpr (KIND == kNormTwo) norm_fold<KIND>(acc, v);
    else top = max(top, magnitude_bits(v));
  }
}

template <int KIND>
__global__ void __launch_bounds__(kThreads)
tensors_norm_kernel(const Tile* __restrict__ tiles, double* __restrict__ partial) {
  pdl_launch_dependents();
  pdl_wait();
  const Tile t = tiles[blockIdx.x];
  double acc = 0.0;
  unsigned top = 0;
  switch (t.types & 15u) {
    case SSGD_F32: tile_norm<KIND>(static_cast<const float*>(t.src), t.n, acc, top); break;
    case SSGD_BF16: tile_norm<KIND>(static_cast<const __nv_bfloat16*>(t.src), t.n, acc, top); break;
    default: tile_norm<KIND>(static_cast<const __half*>(t.src), t.n, acc, top); break;
  }
  __shared__ double part[kThreads / 32];
  const unsigned lane = threadIdx.x & 31u, warp = threadIdx.x >> 5;
  if constexpr (KIND == kNormTwo) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) acc += __shfl_xor_sync(0xFFFFFFFFu, acc, o);
  } else {
    acc = (double)__reduce_max_sync(0xFFFFFFFFu, top);
  }
  if (lane == 0) part[warp] = acc;
  __syncthreads();
  if (threadIdx.x == 0) {
    double s = part[0];
#pragma unroll
    for (int w = 1; w < kThreads / 32; ++w) s = KIND == kNormTwo ? s + part[w] : fmax(s, part[w]);
    partial[blockIdx.x] = s;
  }
}

template <int KIND>
__global__ void __launch_bounds__(kThreads)
norms_finish_kernel(const uint64_t* __restrict__ first_tile, const double* __restrict__ partial, float* __restrict__ norms) {
  pdl_launch_dependents();
  pdl_wait();
  const uint64_t a = first_tile[blockIdx.x], b = first_tile[blockIdx.x + 1];
  double s = 0.0;
  for (uint64_t i = a + threadIdx.x; i < b; i += kThreads) s = KIND == kNormTwo ? s + partial[i] : fmax(s, partial[i]);
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    const double other = __shfl_xor_sync(0xFFFFFFFFu, s, o);
    s = KIND == kNormTwo ? s + other : fmax(s, other);
  }
  __shared__ double part[kThreads / 32];
  if ((threadIdx.x & 31u) == 0) part[threadIdx.x >> 5] = s;
  __syncthreads();
  if (threadIdx.x == 0) {
    double r = part[0];
#pragma unroll
    for (int w = 1; w < kThreads / 32; ++w) r = KIND == kNormTwo ? r + part[w] : fmax(r, part[w]);
    norms[blockIdx.x] = KIND == kNormTwo ? (float)sqrt(r) : __uint_as_float((unsigned)r);
  }
}

// c of one group, and whether its rows are zeroed instead (norm not finite, when the caller asked for that).
__device__ __forceinline__ float clip_factor(float norm, float max_norm, int zero_nonfinite, bool* zero) {
  *zero = zero_nonfinite && !(norm <= 3.402823466e38f);
  return norm > max_norm ? __fdiv_rn(max_norm, norm) : (norm == norm ? 1.0f : norm);
}

template <typename S, typename D>
__device__ __forceinline__ void tile_scale(const S* __restrict__ src, D* __restrict__ dst, unsigned n, float c, bool zero) {
  const bool aligned = ((reinterpret_cast<uintptr_t>(src) & (4 * sizeof(S) - 1)) | (reinterpret_cast<uintptr_t>(dst) & (4 * sizeof(D) - 1))) == 0;
  const unsigned body = aligned ? n & ~3u : 0u;
#pragma unroll 4
  for (unsigned i = threadIdx.x * 4; i < body; i += kThreads * 4) {
    float4 q = load4(src + i);
    q = make_float4(__fmul_rn(q.x, c), __fmul_rn(q.y, c), __fmul_rn(q.z, c), __fmul_rn(q.w, c));
    if (zero) q = make_float4(0.f, 0.f, 0.f, 0.f);
    store4(dst + i, q);
  }
#pragma unroll 4
  for (unsigned i = body + threadIdx.x; i < n; i += kThreads) {
    const float v = __fmul_rn(to_float(src[i]), c);
    dst[i] = from_float<D>(zero ? 0.0f : v);
  }
}

template <typename S>
__device__ __forceinline__ void tile_scale_from(const Tile& t, float c, bool zero) {
  const S* src = static_cast<const S*>(t.src);
  switch (t.types >> 4) {
    case SSGD_F32: tile_scale(src, static_cast<float*>(t.dst), t.n, c, zero); break;
    case SSGD_BF16: tile_scale(src, static_cast<__nv_bfloat16*>(t.dst), t.n, c, zero); break;
    default: tile_scale(src, static_cast<__half*>(t.dst), t.n, c, zero); break;
  }
}

__global__ void __launch_bounds__(kThreads)
tensors_scale_kernel(const Tile* __restrict__ tiles, const float* __restrict__ norms, float max_norm, int zero_nonfinite) {
  pdl_launch_dependents();
  pdl_wait();
  const Tile t = tiles[blockIdx.x];
  if (t.dst == nullptr) return;
  bool zero;
  const float c = clip_factor(norms[t.group], max_norm, zero_nonfinite, &zero);
  if (t.src == t.dst && c == 1.0f && !zero) return;   // in place and nothing to change
  switch (t.types & 15u) {
    case SSGD_F32: tile_scale_from<float>(t, c, zero); break;
    case SSGD_BF16: tile_scale_from<__nv_bfloat16>(t, c, zero); break;
    default: tile_scale_from<__half>(t, c, zero); break;
  }
}

ssgd_status check_tensors(const ssgd_tensor* t, size_t T, size_t groups, size_t* tiles) {
  if (groups < 1 || groups > SSGD_MAX_WORKERS) return SSGD_ERR_SIZE;
  if (T > 0 && !t) return SSGD_ERR_NULL;
  size_t count = 0;
  uint32_t group = 0;
  for (size_t i = 0; i < T; ++i) {
    if (t[i].group >= groups || t[i].group < group) return SSGD_ERR_ARG;
    group = t[i].group;
    const size_t sb = dtype_bytes(t[i].src_type), db = dtype_bytes(t[i].dst_type);
    if (sb == 0 || db == 0) return SSGD_ERR_ARG;
    if (t[i].n == 0) continue;
    if (!t[i].src) return SSGD_ERR_NULL;
    if (reinterpret_cast<uintptr_t>(t[i].src) % sb != 0 || reinterpret_cast<uintptr_t>(t[i].dst) % db != 0) return SSGD_ERR_ALIGN;
    if (t[i].n > ((size_t)1 << 48)) return SSGD_ERR_SIZE;
    count += (t[i].n - 1) / kTile + 1;
    if (count > kMaxGrid) return SSGD_ERR_SIZE;
  }
  *tiles = count;
  return SSGD_OK;
}

ssgd_status check_table(const void* table, size_t tiles, size_t groups, const void* ws, const float* norms) {
  if (!table || !ws || !norms) return SSGD_ERR_NULL;
  if (!aligned16(table) || !aligned16(ws) || (reinterpret_cast<uintptr_t>(norms) & 3u)) return SSGD_ERR_ALIGN;
  if (groups < 1 || groups > SSGD_MAX_WORKERS || tiles > kMaxGrid) return SSGD_ERR_SIZE;
  return SSGD_OK;
}

inline const Tile* table_tiles(const void* table, size_t groups) {
  return reinterpret_cast<const Tile*>(static_cast<const char*>(table) + table_head_bytes(groups));
}

template <int KIND>
void launch_norm(const void* table, size_t tiles, size_t groups, double* ws, float* norms, cudaStream_t s) {
  if (tiles > 0)
    launch_kernel(tensors_norm_kernel<KIND>, dim3((unsigned)tiles), dim3(kThreads), 0, s, true, table_tiles(table, groups), ws);
  launch_kernel(norms_finish_kernel<KIND>, dim3((unsigned)groups), dim3(kThreads), 0, s, true,
                static_cast<const uint64_t*>(table), static_cast<const double*>(ws), norms);
}

}  // namespace

extern "C" {

ssgd_status ssgd_table_size(const ssgd_tensor* tensors, size_t T, size_t groups, size_t* tiles, size_t* table_bytes,
                            size_t* ws_bytes) {
  if (!tiles || !table_bytes || !ws_bytes) return SSGD_ERR_NULL;
  const ssgd_status st = check_tensors(tensors, T, groups, tiles);
  if (st != SSGD_OK) return st;
  *table_bytes = table_head_bytes(groups) + *tiles * sizeof(Tile);
  *ws_bytes = (*tiles + 2) / 2 * 2 * sizeof(double);
  return SSGD_OK;
}

ssgd_status ssgd_table_build(const ssgd_tensor* tensors, size_t T, size_t groups, void* table_host, size_t table_bytes) {
  size_t tiles = 0;
  const ssgd_status st = check_tensors(tensors, T, groups, &tiles);
  if (st != SSGD_OK) return st;
  if (!table_host) return SSGD_ERR_NULL;
  if (table_bytes < table_head_bytes(groups) + tiles * sizeof(Tile)) return SSGD_ERR_SIZE;
  char* base = static_cast<char*>(table_host);
  memset(base, 0, table_head_bytes(groups));
  uint64_t at = 0;
  uint32_t group = 0;
  for (size_t i = 0; i < T; ++i) {
    const size_t sb = dtype_bytes(tensors[i].src_type), db = dtype_bytes(tensors[i].dst_type);
    for (; group < tensors[i].group; ++group) memcpy(base + (group + 1) * sizeof(uint64_t), &at, sizeof at);
    for (size_t o = 0; o < tensors[i].n; o += kTile) {
      Tile e;
      e.src = static_cast<const char*>(tensors[i].src) + o * sb;
      e.dst = tensors[i].dst ? static_cast<char*>(tensors[i].dst) + o * db : nullptr;
      e.n = (uint32_t)(tensors[i].n - o < kTile ? tensors[i].n - o : kTile);
      e.group = tensors[i].group;
      e.types = tensors[i].src_type | tensors[i].dst_type << 4;
      e.unused = 0;
      memcpy(base + table_head_bytes(groups) + at * sizeof(Tile), &e, sizeof e);
      ++at;
    }
  }
  for (; group < groups; ++group) memcpy(base + (group + 1) * sizeof(uint64_t), &at, sizeof at);
  return SSGD_OK;
}

ssgd_status ssgd_tensors_norm(const void* table, size_t tiles, size_t groups, int kind, void* ws, float* norms, void* stream) {
  const ssgd_status st = check_table(table, tiles, groups, ws, norms);
  if (st != SSGD_OK) return st;
  if (kind != SSGD_NORM_TWO && kind != SSGD_NORM_MAX) return SSGD_ERR_ARG;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  if (kind == SSGD_NORM_TWO) launch_norm<kNormTwo>(table, tiles, groups, static_cast<double*>(ws), norms, s);
  else launch_norm<kNormMax>(table, tiles, groups, static_cast<double*>(ws), norms, s);
  return launch_status();
}

ssgd_status ssgd_tensors_clip(const void* table, size_t tiles, size_t groups, int kind, float max_norm, int zero_nonfinite,
                              void* ws, float* norms, void* stream) {
  if (!(max_norm >= 0.0f)) return SSGD_ERR_ARG;
  const ssgd_status st = ssgd_tensors_norm(table, tiles, groups, kind, ws, norms, stream);
  if (st != SSGD_OK || tiles == 0) return st;
  launch_kernel(tensors_scale_kernel, dim3((unsigned)tiles), dim3(kThreads), 0, static_cast<cudaStream_t>(stream), true,
                table_tiles(table, groups), static_cast<const float*>(norms), max_norm, zero_nonfinite);
  return launch_status();
}

}  // extern "C"
