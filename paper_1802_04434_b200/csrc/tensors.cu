// Norm and clipping of gradients that come as many tensors, into the flat rows that the step takes.
// See include/signsgd.h for the contract of each call.
//
// The host cuts every tensor into tiles of at most kTile elements and writes them into a table (caller-owned memory,
// copied to the device once); a CTA takes one tile, so tensors of any number and size are one launch and no CTA gets
// more than its share.  Tiles of a group (a worker) are consecutive.
//   pass 1  tensors_norm_kernel   a sum of squares (or largest magnitude) for each tile
//   pass 2  norms_finish_kernel   norm of each group from its tiles', in a fixed order
//   pass 3  tensors_scale_kernel  dst = c * src with c = max_norm / norm where norm > max_norm, else 1; from the last tile
//                                 to the first, since the last ones read are still in L2
// Small groups: tensors_clip_small_kernel, all of it in one launch, one cluster of eight CTAs for a group.
// Sums go in a fixed order: equal inputs give equal bits.

#include <cooperative_groups.h>
#include <string.h>

#include "host_calls.h"
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

// |v| as ordered bits: NaN sorts above infinity, so one maximum carries it through.
__device__ __forceinline__ unsigned magnitude_bits(float v) { return __float_as_uint(v) & 0x7FFFFFFFu; }

// Squares go to fp64, where the product of two fp32 numbers is exact and neither overflows nor vanishes.
__device__ __forceinline__ void fold8(const float (&v)[8], double& acc) {
#pragma unroll
  for (int i = 0; i < 8; ++i) acc = fma((double)v[i], (double)v[i], acc);
}

// One tile's contribution of this thread: a double for the two-norm, the largest magnitude's bits for the maximum.
template <int KIND, typename T>
__device__ __forceinline__ void tile_norm(const T* __restrict__ src, unsigned n, double& acc, unsigned& top) {
  const unsigned off = (unsigned)(reinterpret_cast<uintptr_t>(src) / sizeof(T)) & 7u;
  const unsigned head = min(n, off ? 8u - off : 0u), groups = (n - head) / 8;
  const T* body = src + head;
  if constexpr (KIND == kNormTwo && sizeof(T) == 2) {
    // Four loads in flight by hand, within the 32 registers of eight CTAs an SM: left to the unrolling there are fewer.  335 M
    // bf16 elements 109 us = 6.2 TB/s; two by hand 137, and that with fours of squares added in fp32 first, which saves
    // three quarters of the conversions to fp64 and was no faster than this even with four (114).
    for (unsigned g0 = threadIdx.x; g0 < groups; g0 += 4 * kThreads) {
      uint4 q[4];
#pragma unroll
      for (int u = 0; u < 4; ++u)
        q[u] = g0 + u * kThreads < groups ? *reinterpret_cast<const uint4*>(body + 8 * (g0 + u * kThreads)) : make_uint4(0, 0, 0, 0);
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        if (g0 + u * kThreads >= groups) break;
        const float v[8] = {low_to_float(T(), q[u].x), high_to_float(T(), q[u].x), low_to_float(T(), q[u].y), high_to_float(T(), q[u].y),
                            low_to_float(T(), q[u].z), high_to_float(T(), q[u].z), low_to_float(T(), q[u].w), high_to_float(T(), q[u].w)};
        fold8(v, acc);
      }
    }
  } else {
#pragma unroll 4
    for (unsigned g = threadIdx.x; g < groups; g += kThreads) {
      float v[8];
      load8(body + 8 * g, v);
      if constexpr (KIND == kNormTwo) {
        fold8(v, acc);
      } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) top = max(top, magnitude_bits(v[i]));
      }
    }
  }
  // what lies before the first and behind the last group of eight: at most 14 elements
  const unsigned rest = head + 8 * groups, loose = n - 8 * groups;
  if (threadIdx.x < loose) {
    const float v = to_float(src[threadIdx.x < head ? threadIdx.x : rest + threadIdx.x - head]);
    if constexpr (KIND == kNormTwo) acc = fma((double)v, (double)v, acc);
    else top = max(top, magnitude_bits(v));
  }
}

template <int KIND>
__device__ __forceinline__ void any_tile_norm(const Tile& t, double& acc, unsigned& top) {
  switch (t.types & 15u) {
    case SSGD_F32: tile_norm<KIND>(static_cast<const float*>(t.src), t.n, acc, top); break;
    case SSGD_BF16: tile_norm<KIND>(static_cast<const __nv_bfloat16*>(t.src), t.n, acc, top); break;
    default: tile_norm<KIND>(static_cast<const __half*>(t.src), t.n, acc, top); break;
  }
}

template <int KIND>
__device__ __forceinline__ double combine(double a, double b) { return KIND == kNormTwo ? a + b : fmax(a, b); }

// Over the CTA, in thread 0 (every thread must call).
template <int KIND, int THREADS>
__device__ __forceinline__ double cta_combine(double s, double* part) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) s = combine<KIND>(s, __shfl_xor_sync(0xFFFFFFFFu, s, o));
  if ((threadIdx.x & 31u) == 0) part[threadIdx.x >> 5] = s;
  __syncthreads();
  double r = part[0];
#pragma unroll
  for (int w = 1; w < THREADS / 32; ++w) r = combine<KIND>(r, part[w]);
  return r;
}

template <int KIND>
__device__ __forceinline__ float finish_norm(double r) { return KIND == kNormTwo ? (float)sqrt(r) : __uint_as_float((unsigned)r); }

template <int KIND>
__global__ void __launch_bounds__(kThreads, 8)
tensors_norm_kernel(const Tile* __restrict__ tiles, double* __restrict__ partial) {
  __shared__ double part[kThreads / 32];
  pdl_launch_dependents();
  pdl_wait();
  const Tile t = tiles[blockIdx.x];
  double acc = 0.0;
  unsigned top = 0;
  any_tile_norm<KIND>(t, acc, top);
  const double s = cta_combine<KIND, kThreads>(KIND == kNormTwo ? acc : (double)top, part);
  if (threadIdx.x == 0) partial[blockIdx.x] = s;
}

constexpr int kFinishThreads = 1024;

template <int KIND>
__global__ void __launch_bounds__(kFinishThreads)
norms_finish_kernel(const uint64_t* __restrict__ first_tile, const double* __restrict__ partial, float* __restrict__ norms) {
  __shared__ double part[kFinishThreads / 32];
  pdl_launch_dependents();
  pdl_wait();
  const uint64_t a = first_tile[blockIdx.x], b = first_tile[blockIdx.x + 1];
  double s = 0.0;
  // sixteen loads in flight: one CTA has to bring a double for every tile of the group
  for (uint64_t i = a + threadIdx.x; i < b; i += 16 * kFinishThreads) {
    double v[16];
#pragma unroll
    for (int u = 0; u < 16; ++u) v[u] = i + u * kFinishThreads < b ? partial[i + u * kFinishThreads] : 0.0;
#pragma unroll
    for (int u = 0; u < 16; ++u) s = combine<KIND>(s, v[u]);
  }
  s = cta_combine<KIND, kFinishThreads>(s, part);
  if (threadIdx.x == 0) norms[blockIdx.x] = finish_norm<KIND>(s);
}

// c of one group, and whether its rows are zeroed instead (norm not finite, when the caller asked for that).  No clipping is a
// copy, whatever the norm.
__device__ __forceinline__ float clip_factor(float norm, float max_norm, int zero_nonfinite, bool* zero) {
  *zero = zero_nonfinite && !(norm <= 3.402823466e38f);
  return norm > max_norm ? __fdiv_rn(max_norm, norm) : (norm == norm || isinf(max_norm) ? 1.0f : norm);
}

// Four elements of a lane at a time where source and destination both allow it, BATCH of them in flight, else element by
// element, LOOSE in flight: lanes lie side by side either way.  In place every element is read before it is written, by
// the thread that writes it.
template <int BATCH, int LOOSE, typename S, typename D>
__device__ __forceinline__ void tile_scale(const S* src, D* dst, unsigned n, float c, bool zero) {
  const bool aligned = ((reinterpret_cast<uintptr_t>(src) & (4 * sizeof(S) - 1)) | (reinterpret_cast<uintptr_t>(dst) & (4 * sizeof(D) - 1))) == 0;
  const unsigned groups = aligned ? n / 4 : 0u;
  for (unsigned g0 = threadIdx.x; g0 < groups; g0 += BATCH * kThreads) {
    float4 v[BATCH];
#pragma unroll
    for (int u = 0; u < BATCH; ++u)
      if (g0 + u * kThreads < groups) v[u] = load4(src + 4 * (g0 + u * kThreads));
#pragma unroll
    for (int u = 0; u < BATCH; ++u)
      if (g0 + u * kThreads < groups) {
        const float4 q = zero ? make_float4(0.f, 0.f, 0.f, 0.f) : make_float4(__fmul_rn(v[u].x, c), __fmul_rn(v[u].y, c), __fmul_rn(v[u].z, c), __fmul_rn(v[u].w, c));
        store4(dst + 4 * (g0 + u * kThreads), q);
      }
  }
  for (unsigned i0 = 4 * groups + threadIdx.x; i0 < n; i0 += LOOSE * kThreads) {
    S v[LOOSE];
#pragma unroll
    for (int u = 0; u < LOOSE; ++u)
      if (i0 + u * kThreads < n) v[u] = src[i0 + u * kThreads];
#pragma unroll
    for (int u = 0; u < LOOSE; ++u)
      if (i0 + u * kThreads < n) dst[i0 + u * kThreads] = from_float<D>(zero ? 0.0f : __fmul_rn(to_float(v[u]), c));
  }
}

template <int BATCH, int LOOSE, typename S>
__device__ __forceinline__ void tile_scale_from(const Tile& t, float c, bool zero) {
  const S* src = static_cast<const S*>(t.src);
  switch (t.types >> 4) {
    case SSGD_F32: tile_scale<BATCH, LOOSE>(src, static_cast<float*>(t.dst), t.n, c, zero); break;
    case SSGD_BF16: tile_scale<BATCH, LOOSE>(src, static_cast<__nv_bfloat16*>(t.dst), t.n, c, zero); break;
    default: tile_scale<BATCH, LOOSE>(src, static_cast<__half*>(t.dst), t.n, c, zero); break;
  }
}

template <int BATCH, int LOOSE>
__device__ __forceinline__ void any_tile_scale(const Tile& t, float norm, float max_norm, int zero_nonfinite) {
  if (t.dst == nullptr) return;
  bool zero;
  const float c = clip_factor(norm, max_norm, zero_nonfinite, &zero);
  if (t.src == t.dst && c == 1.0f && !zero) return;   // in place and nothing to change
  switch (t.types & 15u) {
    case SSGD_F32: tile_scale_from<BATCH, LOOSE, float>(t, c, zero); break;
    case SSGD_BF16: tile_scale_from<BATCH, LOOSE, __nv_bfloat16>(t, c, zero); break;
    default: tile_scale_from<BATCH, LOOSE, __half>(t, c, zero); break;
  }
}

// Bound by memory: 335 M elements in 320 tensors on B200, whole call, fp32 to fp32 584 us = 6.90 TB/s of its three passes, bf16 to
// fp32 415 us = 6.47 TB/s; Resnet-50's 161 tensors x 7 workers in fp32 316 us = 6.80 TB/s.  Measured and worse: batches of 2
// (bf16 442, at 8 CTAs per SM 420), 8 elements a lane (429), half and quarter tiles per CTA (457 - 580), two to four tiles in a
// row per CTA (670 and more), tiles in order instead of from the end (+ 3).
constexpr int kBatch = 4, kLoose = 8;
__global__ void __launch_bounds__(kThreads, 6)
tensors_scale_kernel(const Tile* __restrict__ tiles, const float* __restrict__ norms, float max_norm, int zero_nonfinite) {
  pdl_launch_dependents();
  pdl_wait();
  const Tile t = tiles[gridDim.x - 1 - blockIdx.x];
  any_tile_scale<kBatch, kLoose>(t, norms[t.group], max_norm, zero_nonfinite);
}

// Both passes for groups of few tiles: the cluster's CTAs take the group's tiles in turn, exchange their sums through
// shared memory and scale the same tiles.  SCALE = false: the norms only.
constexpr unsigned kCluster = 8;

template <int KIND, bool SCALE>
__global__ void __launch_bounds__(kThreads)
tensors_clip_small_kernel(const uint64_t* __restrict__ first_tile, const Tile* __restrict__ tiles, float* __restrict__ norms, float max_norm,
                          int zero_nonfinite) {
  __shared__ double part[kThreads / 32];
  __shared__ double mine;
  namespace cg = cooperative_groups;
  cg::cluster_group cluster = cg::this_cluster();
  const unsigned group = blockIdx.x / kCluster, rank = cluster.block_rank();
  pdl_launch_dependents();
  pdl_wait();
  const uint64_t a = first_tile[group], b = first_tile[group + 1];
  double acc = 0.0;
  unsigned top = 0;
  for (uint64_t i = a + rank; i < b; i += kCluster) any_tile_norm<KIND>(tiles[i], acc, top);
  const double s = cta_combine<KIND, kThreads>(KIND == kNormTwo ? acc : (double)top, part);
  if (threadIdx.x == 0) mine = s;
  cluster.sync();
  double all = 0.0;
#pragma unroll
  for (unsigned r = 0; r < kCluster; ++r) all = combine<KIND>(all, *cluster.map_shared_rank(&mine, r));
  const float norm = finish_norm<KIND>(all);
  if (rank == 0 && threadIdx.x == 0) norms[group] = norm;
  if (SCALE)
    for (uint64_t i = a + rank; i < b; i += kCluster) any_tile_scale<2, 4>(tiles[i], norm, max_norm, zero_nonfinite);
  cluster.sync();                                     // nobody leaves while its sum is still read
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

// Workspace: a double for each tile.
inline size_t ws_size(size_t tiles) { return (tiles + 2) / 2 * 2 * sizeof(double); }

// The one-launch form: a tile for each CTA of a cluster on average, no more clusters than are there at one time, and a bound
// on what one group may have if the tiles are not spread evenly.  B200, one launch / three, us, bf16 to fp32: a group of 8
// tiles 4.9 / 5.8, of 16 7.5 / 5.8, of 32 12.6 / 5.9; 15 groups of 1 to 4 tiles 5.0 / 6.2, 16 groups 9.0 / 6.1.
constexpr size_t kSmallTiles = 32, kSmallGroups = 15;
inline bool in_one_launch(size_t tiles, size_t groups) { return groups <= kSmallGroups && tiles <= kSmallTiles && tiles <= groups * kCluster; }

template <int KIND>
ssgd_status launch_clip(const void* table, size_t tiles, size_t groups, bool scale, float max_norm, int zero_nonfinite, void* ws, float* norms,
                        cudaStream_t s) {
  const uint64_t* first = static_cast<const uint64_t*>(table);
  const Tile* list = table_tiles(table, groups);
  if (in_one_launch(tiles, groups)) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)groups * kCluster);
    cfg.blockDim = dim3(kThreads);
    cfg.stream = s;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = kCluster;
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 2;
    auto kernel = scale ? tensors_clip_small_kernel<KIND, true> : tensors_clip_small_kernel<KIND, false>;
    (void)cudaLaunchKernelEx(&cfg, kernel, first, list, norms, max_norm, zero_nonfinite);
    return launch_status();
  }
  double* partial = static_cast<double*>(ws);
  if (tiles > 0) launch_kernel(tensors_norm_kernel<KIND>, dim3((unsigned)tiles), dim3(kThreads), 0, s, true, list, partial);
  launch_kernel(norms_finish_kernel<KIND>, dim3((unsigned)groups), dim3(kFinishThreads), 0, s, true, first, static_cast<const double*>(partial), norms);
  if (scale && tiles > 0)
    launch_kernel(tensors_scale_kernel, dim3((unsigned)tiles), dim3(kThreads), 0, s, true, list, static_cast<const float*>(norms), max_norm, zero_nonfinite);
  return launch_status();
}

}  // namespace

extern "C" {

ssgd_status ssgd_table_size(const ssgd_tensor* tensors, size_t T, size_t groups, size_t* tiles, size_t* table_bytes,
                            size_t* ws_bytes) {
  if (!tiles || !table_bytes || !ws_bytes) return SSGD_ERR_NULL;
  const ssgd_status st = check_tensors(tensors, T, groups, tiles);
  if (st != SSGD_OK) return st;
  *table_bytes = table_head_bytes(groups) + *tiles * sizeof(Tile);
  *ws_bytes = ws_size(*tiles);
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
  return kind == SSGD_NORM_TWO ? launch_clip<kNormTwo>(table, tiles, groups, false, 0.0f, 0, ws, norms, s)
                               : launch_clip<kNormMax>(table, tiles, groups, false, 0.0f, 0, ws, norms, s);
}

ssgd_status ssgd_tensors_clip(const void* table, size_t tiles, size_t groups, int kind, float max_norm, int zero_nonfinite,
                              void* ws, float* norms, void* stream) {
  const ssgd_status st = check_table(table, tiles, groups, ws, norms);
  if (st != SSGD_OK) return st;
  if ((kind != SSGD_NORM_TWO && kind != SSGD_NORM_MAX) || !(max_norm >= 0.0f)) return SSGD_ERR_ARG;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  return kind == SSGD_NORM_TWO ? launch_clip<kNormTwo>(table, tiles, groups, true, max_norm, zero_nonfinite, ws, norms, s)
                               : launch_clip<kNormMax>(table, tiles, groups, true, max_norm, zero_nonfinite, ws, norms, s);
}

ssgd_status ssgd_tensors_clip_block(const uint64_t* a) {
  if (!a) return SSGD_ERR_NULL;
  double max_norm;
  memcpy(&max_norm, a + 4, sizeof max_norm);
  return ssgd_tensors_clip(block_ptr<const void>(a[0]), a[1], a[2], (int)a[3], (float)max_norm, (int)a[5], block_ptr<void>(a[6]),
                           block_ptr<float>(a[7]), block_ptr<void>(a[8]));
}

}  // extern "C"
