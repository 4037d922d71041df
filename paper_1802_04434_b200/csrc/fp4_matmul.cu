// Product of two microscaled 4-bit operands, out[i][j] = tA tB sum_k A[i][k] B[j][k].  See include/signsgd.h.
//
// The tensor cores multiply 4-bit values and apply the block scales themselves (tcgen05.mma, block-scaled): a CTA keeps a
// tile of 128 rows of B by NT rows of A as fp32 accumulators in tensor memory.  B's rows are the accumulator's lanes, so
// a warp's 32 lanes hold 32 neighbours of one row of out and the stores need no transposition; and few rows of A (a
// handful of tokens against a weight) only make NT small, the weight streams through once either way.
//
//   warp 0      one thread brings a stage, 256 of k: 128 x 128 and NT x 128 bytes of codes (tiled copies, 128-byte
//               swizzle, out-of-range rows and columns filled with zero codes) and their scale tiles (bulk copies)
//   warp 1      one thread copies the scales into tensor memory and issues four MMAs of 64 of k per stage
//   warps 2..5  read the accumulators and write out
// Every stage has scale columns of its own, so that nothing is overwritten before the commit that frees the stage.
// Few output tiles: a cluster of 2, 4 or 8 CTAs splits k, the partial tiles meet in shared memory and each CTA adds up
// its share of the columns over the cluster, in rank order: no atomics, equal inputs give equal bits.

#include <cooperative_groups.h>

#include "host_common.h"
#include "dtypes.cuh"
#include "fp4.cuh"
#include "sm100.cuh"

namespace {

constexpr int kMmaThreads = 192;
constexpr unsigned kTileJ = 128;            // rows of B in a tile: lanes of the accumulator
constexpr unsigned kPolls = 200000;         // bound of a wait, about 0.2 s

template <int FORMAT, int NT>
struct Shape {
  static constexpr unsigned blocks = FORMAT == SSGD_MXFP4 ? 2 : 4;          // scale tiles (of four blocks) of a stage and 128 rows
  static constexpr unsigned row_tiles = (NT + 127) / 128;                  // of A
  static constexpr unsigned b_bytes = kTileJ * 128, a_bytes = NT * 128;
  static constexpr unsigned scale_bytes = blocks * 512;
  static constexpr unsigned stage_bytes = b_bytes + a_bytes + ((1 + row_tiles) * scale_bytes + 1023) / 1024 * 1024;
  static constexpr unsigned stages = 221184 / stage_bytes < 8 ? 221184 / stage_bytes : 8;
  static constexpr unsigned scale_columns = (1 + row_tiles) * blocks * 4;  // of a stage, in tensor memory
  static constexpr unsigned columns_used = NT + stages * scale_columns;
  static constexpr unsigned columns = columns_used <= 64 ? 64 : columns_used <= 128 ? 128 : columns_used <= 256 ? 256 : 512;
  static_assert(columns_used <= 512, "tensor memory");
  static_assert(NT * kTileJ * 4 <= stages * stage_bytes, "the partial tile reuses the stages");
  // One CTA per SM always: two clusters whose CTAs hold and wait for tensor memory on each other's SMs would never end.
  static constexpr unsigned smem = (stages * stage_bytes < 118784 ? 118784 : stages * stage_bytes) + 1024;
};

struct ProductArgs {
  const uint8_t* a_scales;
  const uint8_t* b_scales;
  const float* a_ts;
  const float* b_ts;
  void* out;
  unsigned* status;
  size_t ldo;
  unsigned M, N;
  unsigned k_chunks;      // 64-column pieces of k
  unsigned tiles_k;       // scale tiles along k of one row of tiles
  unsigned a_row_tiles;   // scale row tiles of A
  unsigned tiles_i;
  int dtype;
};

__device__ __forceinline__ void store_out(const ProductArgs& p, size_t at, float v) {
  if (p.dtype == SSGD_F32) static_cast<float*>(p.out)[at] = v;
  else if (p.dtype == SSGD_BF16) static_cast<__nv_bfloat16*>(p.out)[at] = __float2bfloat16_rn(v);
  else static_cast<__half*>(p.out)[at] = __float2half_rn(v);
}

template <int FORMAT, int NT>
__global__ void __launch_bounds__(kMmaThreads, 1)
fp4_matmul_kernel(const __grid_constant__ CUtensorMap a_map, const __grid_constant__ CUtensorMap b_map, const ProductArgs p) {
  using S = Shape<FORMAT, NT>;
  extern __shared__ unsigned char dynamic_smem[];
  __shared__ __align__(8) uint64_t bars[2 * S::stages + 1];
  __shared__ unsigned tmem_base, failed;
  namespace cg = cooperative_groups;
  cg::cluster_group cluster = cg::this_cluster();
  const unsigned splits = cluster.num_blocks(), split = cluster.block_rank();
  unsigned char* stage_mem = dynamic_smem + ((1024u - (smem_u32(dynamic_smem) & 1023u)) & 1023u);
  const unsigned stage0 = smem_u32(stage_mem);
  const unsigned full = smem_u32(bars), empty = full + 8 * S::stages, done = empty + 8 * S::stages;
  const unsigned warp = threadIdx.x >> 5, lane = threadIdx.x & 31u;

  const unsigned tile = blockIdx.x / splits;
  const unsigned i0 = tile % p.tiles_i * NT, j0 = tile / p.tiles_i * kTileJ;
  const unsigned stages_k = (p.k_chunks + 3) / 4;
  const unsigned first = (unsigned)((uint64_t)stages_k * split / splits), last = (unsigned)((uint64_t)stages_k * (split + 1) / splits);

  if (threadIdx.x == 0) {
    prefetch_tensor_map(&a_map);
    prefetch_tensor_map(&b_map);
    for (unsigned s = 0; s < S::stages; ++s) {
      mbarrier_init(full + 8 * s, 1);
      mbarrier_init(empty + 8 * s, 1);
    }
    mbarrier_init(done, 1);
    mbarrier_init_fence();
    failed = 0;
  }
  pdl_launch_dependents();
  pdl_wait();                                   // before tensor memory is taken: its last holder has finished
  if (warp == 1) tmem_alloc(smem_u32(&tmem_base), S::columns);
  tcgen05_fence_before();
  __syncthreads();
  tcgen05_fence_after();
  const unsigned tmem = tmem_base;
  bool ok = true;
  unsigned issued = 0;                          // stages that this thread has asked for

  if (warp == 0) {
    if (lane == 0) {
      const unsigned jt = j0 / 128, it = i0 / 128;
      for (unsigned k = first; k < last && ok; ++k) {
        const unsigned n = k - first, s = n % S::stages;
        if (n >= S::stages) ok = mbarrier_wait(empty + 8 * s, (n / S::stages - 1) & 1u, kPolls);
        if (!ok) break;
        const unsigned base = stage0 + s * S::stage_bytes, bar = full + 8 * s;
        const unsigned kt = k * S::blocks, blocks = min(S::blocks, p.tiles_k - kt);
        const unsigned row_tiles = min(S::row_tiles, p.a_row_tiles - it);
        issued = n + 1;
        mbarrier_expect(bar, S::b_bytes + S::a_bytes + (1 + row_tiles) * blocks * 512);
        tma_load_2d(base, &b_map, (int)(k * 128), (int)j0, bar);
        tma_load_2d(base + S::b_bytes, &a_map, (int)(k * 128), (int)i0, bar);
        const unsigned sc = base + S::b_bytes + S::a_bytes;
        bulk_copy(sc, p.b_scales + ((size_t)jt * p.tiles_k + kt) * 512, blocks * 512, bar);
        for (unsigned t = 0; t < row_tiles; ++t)
          bulk_copy(sc + (1 + t) * S::scale_bytes, p.a_scales + ((size_t)(it + t) * p.tiles_k + kt) * 512, blocks * 512, bar);
      }
    }
  } else if (warp == 1) {
    if (lane == 0) {
      for (unsigned k = first; k < last && ok; ++k) {
        const unsigned n = k - first, s = n % S::stages;
        ok = mbarrier_wait(full + 8 * s, (n / S::stages) & 1u, kPolls);
        if (!ok) break;
        tcgen05_fence_after();
        const unsigned base = stage0 + s * S::stage_bytes, sc = base + S::b_bytes + S::a_bytes;
        const unsigned columns = tmem + NT + s * S::scale_columns;
        const unsigned chunks = min(4u, p.k_chunks - k * 4), blocks = min(S::blocks, p.tiles_k - k * S::blocks);
        // scales: 4 columns for each tile of 128 rows x 4 blocks; B's, then for each four blocks A's row tiles side by side
        for (unsigned q = 0; q < blocks; ++q) {
          tcgen05_copy_scales(columns + q * 4, smem_descriptor(sc + q * 512, 128, 0));
          for (unsigned t = 0; t < S::row_tiles; ++t)
            tcgen05_copy_scales(columns + S::blocks * 4 + (q * S::row_tiles + t) * 4, smem_descriptor(sc + (1 + t) * S::scale_bytes + q * 512, 128, 0));
        }
        const uint64_t b_desc = smem_descriptor(base, 1024, 2), a_desc = smem_descriptor(base + S::b_bytes, 1024, 2);
        for (unsigned c = 0; c < chunks; ++c) {
          const unsigned q = FORMAT == SSGD_MXFP4 ? c / 2 : c, id = FORMAT == SSGD_MXFP4 ? (c & 1u) * 2 : 0;
          mma_fp4<FORMAT == SSGD_MXFP4>(tmem, b_desc + 2 * c, a_desc + 2 * c, mma_fp4_descriptor(kTileJ, NT, FORMAT == SSGD_MXFP4, id),
                                        columns + q * 4, columns + S::blocks * 4 + q * S::row_tiles * 4, n > 0 || c > 0);
        }
        tcgen05_commit(empty + 8 * s);
      }
      if (!ok) atomicExch(&failed, 1u);        // the epilogue looks at it once `done` has come
      tcgen05_commit(done);
    }
  } else {
    ok = mbarrier_wait(done, 0, 4 * kPolls + 64 * (last - first)) && *(volatile unsigned*)&failed == 0;
    tcgen05_fence_after();
    const unsigned quarter = warp & 3u, j = j0 + quarter * 32 + lane;
    const unsigned lanes = tmem + (quarter << 21);
    const float ts = (p.a_ts ? __ldg(p.a_ts) : 1.0f) * (p.b_ts ? __ldg(p.b_ts) : 1.0f);
    float* partial = reinterpret_cast<float*>(stage_mem);       // [NT][128]; the stages are used up by now
    if (ok) {
#pragma unroll 1
      for (unsigned c = 0; c < NT; c += 16) {
        if (i0 + c >= p.M) break;
        unsigned v[16];
        tmem_load16(lanes + c, v);
        tmem_load_wait(v);
        if (splits == 1) {
#pragma unroll
          for (unsigned q = 0; q < 16; ++q)
            if (i0 + c + q < p.M && j < p.N) store_out(p, (size_t)(i0 + c + q) * p.ldo + j, __uint_as_float(v[q]) * ts);
        } else {
#pragma unroll
          for (unsigned q = 0; q < 16; ++q) partial[(c + q) * kTileJ + quarter * 32 + lane] = __uint_as_float(v[q]);
        }
      }
      tcgen05_fence_before();
    }
  }
  if (!ok) atomicExch(&failed, 1u);
  __syncwarp();
  __syncthreads();
  if (failed) {
    // copies that were asked for have to land before the CTA gives its memory up
    if (threadIdx.x == 0) {
      atomicOr(p.status, 1u);
      for (unsigned n = issued > S::stages ? issued - S::stages : 0; n < issued; ++n)
        (void)mbarrier_wait(full + 8 * (n % S::stages), (n / S::stages) & 1u, kPolls);
    }
    __syncthreads();
  }
  if (splits > 1) {
    __syncwarp();
    cluster.sync();
    if (warp >= 2) {
      const unsigned row = (warp & 3u) * 32 + lane, j = j0 + row;
      const float ts = (p.a_ts ? __ldg(p.a_ts) : 1.0f) * (p.b_ts ? __ldg(p.b_ts) : 1.0f);
      float* partial = reinterpret_cast<float*>(stage_mem);
      for (unsigned c = split; c < NT && i0 + c < p.M; c += splits) {
        float v = 0.0f;
        for (unsigned r = 0; r < splits; ++r) v += cluster.map_shared_rank(partial, r)[c * kTileJ + row];
        if (j < p.N) store_out(p, (size_t)(i0 + c) * p.ldo + j, v * ts);
      }
    }
    __syncwarp();
    cluster.sync();                             // nobody leaves while its shared memory is still read
  }
  if (warp == 1) {
    tcgen05_fence_after();
    tmem_free(tmem, S::columns);
  }
}

// cuTensorMapEncodeTiled, found through the runtime so that the library needs no link to the driver.
typedef CUresult (*EncodeTiled)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*,
                                const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle,
                                CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
EncodeTiled encode_tiled() {
  static EncodeTiled cached = nullptr;          // any thread stores the same value
  EncodeTiled f = __atomic_load_n(&cached, __ATOMIC_RELAXED);
  if (f) return f;
  void* p = nullptr;
  cudaDriverEntryPointQueryResult found;
  if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &p, 12000, cudaEnableDefault, &found) != cudaSuccess ||
      found != cudaDriverEntryPointSuccess)
    return nullptr;
  f = reinterpret_cast<EncodeTiled>(p);
  __atomic_store_n(&cached, f, __ATOMIC_RELAXED);
  return f;
}

// Codes as a byte matrix, in boxes of 128 bytes x `box_rows`, 128-byte swizzle, zero beyond the edges.
bool code_map(CUtensorMap* map, const uint8_t* codes, size_t rows, size_t row_bytes, unsigned box_rows) {
  const EncodeTiled f = encode_tiled();
  if (!f) return false;
  const cuuint64_t dims[2] = {row_bytes, rows}, strides[1] = {row_bytes};
  const cuuint32_t box[2] = {128, box_rows}, steps[2] = {1, 1};
  return f(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, const_cast<uint8_t*>(codes), dims, strides, box, steps, CU_TENSOR_MAP_INTERLEAVE_NONE,
           CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <int FORMAT, int NT>
ssgd_status launch_product(const CUtensorMap& a_map, const CUtensorMap& b_map, const ProductArgs& p, unsigned tiles, unsigned splits, cudaStream_t s) {
  using S = Shape<FORMAT, NT>;
  auto kernel = fp4_matmul_kernel<FORMAT, NT>;
  if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)S::smem) != cudaSuccess) return SSGD_ERR_CUDA;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(tiles * splits);
  cfg.blockDim = dim3(kMmaThreads);
  cfg.dynamicSmemBytes = S::smem;
  cfg.stream = s;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = splits;
  attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 2;
  (void)cudaLaunchKernelEx(&cfg, kernel, a_map, b_map, p);
  return launch_status();
}

template <int FORMAT>
ssgd_status product(const uint8_t* a, const uint8_t* as, const float* ats, const uint8_t* b, const uint8_t* bs, const float* bts, size_t M,
                    size_t N, size_t K, void* out, int dtype, size_t ldo, unsigned* status, cudaStream_t s) {
  DeviceInfo info;
  if (!device_info(&info)) return SSGD_ERR_CUDA;
  const size_t row_bytes = ssgd_fp4_row_bytes(K);
  // widest tile that A's rows fill, 256 only where it still leaves every SM a tile
  const size_t tiles_j = (N + kTileJ - 1) / kTileJ;
  unsigned nt = M <= 16 ? 16 : M <= 32 ? 32 : M <= 64 ? 64 : M <= 128 ? 128 : 256;
  const size_t tiles_i = (M + nt - 1) / nt;
  if (tiles_j * tiles_i > (size_t)1 << 27) return SSGD_ERR_SIZE;
  const unsigned tiles = (unsigned)(tiles_j * tiles_i);
  const unsigned stages_k = (unsigned)((row_bytes + 127) / 128);
  unsigned splits = 1;
  while (splits < 8 && tiles * splits * 2 <= (unsigned)info.sms && splits * 2 <= stages_k) splits *= 2;
  CUtensorMap a_map, b_map;
  if (!code_map(&a_map, a, M, row_bytes, nt) || !code_map(&b_map, b, N, row_bytes, kTileJ)) return SSGD_ERR_CUDA;
  ProductArgs p;
  p.a_scales = as; p.b_scales = bs; p.a_ts = ats; p.b_ts = bts; p.out = out; p.status = status; p.ldo = ldo;
  p.M = (unsigned)M; p.N = (unsigned)N;
  p.k_chunks = (unsigned)((row_bytes + 31) / 32);
  p.tiles_k = (unsigned)((fp4_block_count(FORMAT, K) + 3) / 4);
  p.a_row_tiles = (unsigned)((M + 127) / 128);
  p.tiles_i = (unsigned)tiles_i;
  p.dtype = dtype;
  switch (nt) {
    case 16: return launch_product<FORMAT, 16>(a_map, b_map, p, tiles, splits, s);
    case 32: return launch_product<FORMAT, 32>(a_map, b_map, p, tiles, splits, s);
    case 64: return launch_product<FORMAT, 64>(a_map, b_map, p, tiles, splits, s);
    case 128: return launch_product<FORMAT, 128>(a_map, b_map, p, tiles, splits, s);
    default: return launch_product<FORMAT, 256>(a_map, b_map, p, tiles, splits, s);
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
  if (K == 0) {
    const size_t e = dtype_bytes((unsigned)dtype);
    return cudaMemset2DAsync(out, ldo * e, 0, N * e, M, s) == cudaSuccess ? SSGD_OK : SSGD_ERR_CUDA;
  }
  return format == SSGD_MXFP4
             ? product<SSGD_MXFP4>(a_codes, a_scales, a_tensor_scale, b_codes, b_scales, b_tensor_scale, M, N, K, out, dtype, ldo, status, s)
             : product<SSGD_NVFP4>(a_codes, a_scales, a_tensor_scale, b_codes, b_scales, b_tensor_scale, M, N, K, out, dtype, ldo, status, s);
}

}  // extern "C"
