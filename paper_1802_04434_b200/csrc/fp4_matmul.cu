// Product of two microscaled 4-bit operands, out[i][j] = tA tB sum_k A[i][k] B[j][k].  See include/signsgd.h.
//
// The tensor cores multiply 4-bit values and apply the block scales themselves (tcgen05.mma, block-scaled): products and
// scales are exact, sums are fp32.  Two kernels:
//
// fp4_matmul_kernel, up to 128 rows of A: a CTA keeps a tile of 128 rows of B by NT rows of A as fp32 accumulators in
// tensor memory.  B's rows are the accumulator's lanes, so a warp's 32 lanes hold 32 neighbours of one row of out and the
// stores need no transposition; and few rows of A (a handful of tokens against a weight) only make NT small, the weight
// streams through once either way.
//   warp 0      one thread brings a stage, 256 of k: 128 x 128 and NT x 128 bytes of codes (tiled copies, 128-byte
//               swizzle, out-of-range rows and columns filled with zero codes) and their scale tiles (bulk copies)
//   warp 1      one thread copies the scales into tensor memory and issues four MMAs of 64 of k per stage
//   warps 2..9  read the accumulators and write out, two warps to a quarter of the lanes, 32 columns in turn
// Every stage has scale columns of its own, so that nothing is overwritten before the commit that frees the stage.
// Few output tiles: a cluster of 2, 4 or 8 CTAs splits k, the partial tiles meet in shared memory and each CTA adds up
// its share of the columns over the cluster, in rank order: no atomics, equal inputs give equal bits.
// Bound by the weight's bytes (B200: 16 rows against 18944 x 8192 9.7 us = 8.5 TB/s from L2 and HBM); a small one by its
// launch and one trip to memory (one row against 4096 x 1024: 3.6 us).
//
// fp4_matmul_pair_kernel, more rows: below.  B200, 8192^3 to bf16, a few in a row: mx 184 us = 5980 TFLOP/s, nv 203 us = 5420 (four
// times the library's measured bf16 rate, 1666, is 6664).  The same MMAs on operands that are not loaded again take 150 / 162
// us: the rest is bytes from L2 to shared memory.  Run for longer it is bound by power: 234 us nv at 1.37 GHz and 945 W.

#include <cooperative_groups.h>

#include "host_calls.h"
#include "dtypes.cuh"
#include "fp4.cuh"
#include "sm100.cuh"

namespace {

constexpr int kMmaThreads = 320;            // copies, MMAs, eight warps that write out
constexpr unsigned kTileJ = 128;            // rows of B in a tile: lanes of the accumulator
constexpr unsigned kPolls = 200000;         // bound of a wait, about 0.2 s
// Bits of a partial sum that a CTA could not finish: a NaN that no arithmetic makes, looked for where the cluster's sum is NaN.
// (A flag of each CTA, asked for through the cluster's shared memory, costs 0.2 us of a split product's 4 us, this 0.05.)
constexpr unsigned kGivenUp = 0x7FC0DEADu;

// One stage's tensor-core work: its scales to tensor memory (4 columns for each tile of 128 rows x 4 blocks: the lanes'
// operand first, then for each four blocks the columns' operand's row tiles side by side), then up to four MMAs of 64 of k.
// Unrolled throughout: a loop over them costs the issuing thread more than the tensor cores take (B200: 530 clocks a
// stage instead of 356 at NT = 64).
//   p_desc, q_desc  codes of the lanes' and the columns' operand;  sc_desc  scale tiles, the columns' operand's behind
//   half            column at which the scales of the columns' operand begin in their tile
template <int FORMAT, int NT, bool PAIR>
__device__ __forceinline__ void issue_stage(unsigned d, uint64_t p_desc, uint64_t q_desc, uint64_t sc_desc, unsigned columns, unsigned half,
                                            unsigned chunks, bool first) {
  constexpr bool kE8M0 = FORMAT == SSGD_MXFP4;
  constexpr unsigned blocks = kE8M0 ? 2 : 4, row_tiles = (NT + 127) / 128;
#pragma unroll
  for (unsigned q = 0; q < blocks; ++q) {
#pragma unroll
    for (unsigned t = 0; t <= row_tiles; ++t) {
      const unsigned to = columns + (t == 0 ? q * 4 : blocks * 4 + (q * row_tiles + t - 1) * 4);
      if (PAIR) tcgen05_copy_scales_pair(to, sc_desc + (t * blocks + q) * 32);
      else tcgen05_copy_scales(to, sc_desc + (t * blocks + q) * 32);
    }
  }
#pragma unroll
  for (unsigned c = 0; c < 4; ++c) {
    const unsigned q = kE8M0 ? c / 2 : c, id = kE8M0 ? (c & 1u) * 2 : 0;
    const unsigned idesc = mma_fp4_descriptor(PAIR ? 256 : 128, NT, kE8M0, id), ps = columns + q * 4, qs = columns + blocks * 4 + q * row_tiles * 4 + half;
    if (c == 0 || c < chunks) {
      if (PAIR) mma_fp4_pair<kE8M0>(d, p_desc + 2 * c, q_desc + 2 * c, idesc, ps, qs, c > 0 || !first);
      else mma_fp4<kE8M0>(d, p_desc + 2 * c, q_desc + 2 * c, idesc, ps, qs, c > 0 || !first);
    }
  }
}

template <int FORMAT, int NT>
struct Shape {
  static constexpr unsigned blocks = FORMAT == SSGD_MXFP4 ? 2 : 4;          // scale tiles (of four blocks) of a stage and 128 rows
  static_assert(NT <= 128, "one scale tile holds A's rows");
  static constexpr unsigned b_bytes = kTileJ * 128, a_bytes = NT * 128;
  static constexpr unsigned scale_bytes = blocks * 512;
  static constexpr unsigned stage_bytes = b_bytes + a_bytes + (2 * scale_bytes + 1023) / 1024 * 1024;
  static constexpr unsigned stages = 221184 / stage_bytes < 8 ? 221184 / stage_bytes : 8;
  static constexpr unsigned scale_columns = 2 * blocks * 4;               // of a stage, in tensor memory
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
  unsigned tiles_i;
  unsigned starve;        // bytes that a stage waits for in vain: 0 but in the self-test of the waits
};

// The tensor scales of both operands.  Powers of two up to 2^120 either way, so their product may leave fp32's range where the
// result does not, or is an exact zero: then they multiply one after the other.  Both are large, or both small, in that
// case, so that the first multiplication does not leave the range unless the result does; where their product is in range
// that would not be so (2^117 and 2^-100).  The second multiplication of all results would cost 8 % of a product that writes
// much (8192 x 8192 x 256 to bf16 25.3 -> 27.5 us), so the first is a branch that is hardly ever taken (25.5, nv 25.8 us).
struct TensorScales { float first, last; };
__device__ __forceinline__ TensorScales tensor_scales(const float* a, const float* b) {
  const float ta = a ? __ldg(a) : 1.0f, tb = b ? __ldg(b) : 1.0f, both = ta * tb;
  const bool in_range = fabsf(both) >= 1.175494351e-38f && fabsf(both) <= 3.402823466e38f;
  return in_range ? TensorScales{1.0f, both} : TensorScales{ta, tb};
}
// 32 accumulators times the first of them.
__device__ __forceinline__ void scale_first(unsigned (&v)[32], const TensorScales& t) {
  if (__builtin_expect(t.first != 1.0f, 0)) {
#pragma unroll
    for (unsigned q = 0; q < 32; ++q) v[q] = __float_as_uint(__uint_as_float(v[q]) * t.first);
  }
}

// 32 accumulators of one lane to a column of out (rows of stride ldo), `left` of them wanted.
template <typename T>
__device__ __forceinline__ void store_column(T* o, size_t ldo, const unsigned (&v)[32], unsigned left, float ts) {
  if (left >= 32) {
#pragma unroll
    for (unsigned q = 0; q < 32; ++q) o[q * ldo] = from_float<T>(__uint_as_float(v[q]) * ts);
  } else {
#pragma unroll
    for (unsigned q = 0; q < 32; ++q)
      if (q < left) o[q * ldo] = from_float<T>(__uint_as_float(v[q]) * ts);
  }
}

template <int FORMAT, int NT, typename T>
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
    if (elect_one()) {
      const unsigned jt = j0 / 128, it = i0 / 128;
      for (unsigned k = first; k < last && ok; ++k) {
        const unsigned n = k - first, s = n % S::stages;
        if (n >= S::stages) ok = mbarrier_wait(empty + 8 * s, (n / S::stages - 1) & 1u, kPolls);
        if (!ok) break;
        const unsigned base = stage0 + s * S::stage_bytes, bar = full + 8 * s;
        const unsigned kt = k * S::blocks, blocks = min(S::blocks, p.tiles_k - kt);
        issued = n + 1;
        mbarrier_expect(bar, S::b_bytes + S::a_bytes + 2 * blocks * 512 + p.starve);
        tma_load_2d(base, &b_map, (int)(k * 128), (int)j0, bar);
        tma_load_2d(base + S::b_bytes, &a_map, (int)(k * 128), (int)i0, bar);
        const unsigned sc = base + S::b_bytes + S::a_bytes;
        bulk_copy(sc, p.b_scales + ((size_t)jt * p.tiles_k + kt) * 512, blocks * 512, bar);
        bulk_copy(sc + S::scale_bytes, p.a_scales + ((size_t)it * p.tiles_k + kt) * 512, blocks * 512, bar);
      }
    }
  } else if (warp == 1) {
    if (elect_one()) {
      const uint64_t p_desc = smem_descriptor(stage0, 1024, 2), q_desc = smem_descriptor(stage0 + S::b_bytes, 1024, 2),
                     sc_desc = smem_descriptor(stage0 + S::b_bytes + S::a_bytes, 128, 0);
      bool ready = false;                       // the stage's operands are known to be there
      for (unsigned k = first, s = 0, parity = 0; k < last; ++k) {
        ok = ready || mbarrier_wait(full + 8 * s, parity, kPolls);
        if (!ok) break;
        tcgen05_fence_after();
        const unsigned next = s + 1 == S::stages ? 0 : s + 1, next_parity = parity ^ (next == 0);
        ready = mbarrier_test(full + 8 * next, next_parity);      // its answer comes while this stage is issued
        const unsigned at = s * (S::stage_bytes >> 4);
        issue_stage<FORMAT, NT, false>(tmem, p_desc + at, q_desc + at, sc_desc + at, tmem + NT + s * S::scale_columns, 0, p.k_chunks - k * 4, k == first);
        tcgen05_commit(empty + 8 * s);
        s = next;
        parity = next_parity;
      }
      if (!ok) atomicExch(&failed, 1u);        // the epilogue looks at it once `done` has come
      tcgen05_commit(done);
    }
  } else {
    ok = mbarrier_wait(done, 0, 4 * kPolls + 64 * (last - first)) && *(volatile unsigned*)&failed == 0;
    tcgen05_fence_after();
    const unsigned quarter = warp & 3u, j = j0 + quarter * 32 + lane;
    const unsigned lanes = tmem + (quarter << 21);
    const TensorScales ts = tensor_scales(p.a_ts, p.b_ts);
    float* partial = reinterpret_cast<float*>(stage_mem);       // [NT][128]; the stages are used up by now
    if (ok) {
#pragma unroll 1
      for (unsigned c = (warp >= 6) * 32; c < NT; c += 64) {
        if (i0 + c >= p.M) break;
        unsigned v[32];
        tmem_read32(lanes + c, v);                              // at NT = 16 the columns from 16 on are other data, not wanted
        const unsigned left = min((unsigned)NT - c, p.M - (i0 + c));
        if (splits == 1) {
          scale_first(v, ts);
          if (j < p.N) store_column(static_cast<T*>(p.out) + (size_t)(i0 + c) * p.ldo + j, p.ldo, v, left, ts.last);
        } else {
#pragma unroll
          for (unsigned q = 0; q < 32; ++q)
            if (q < left) partial[(c + q) * kTileJ + quarter * 32 + lane] = __uint_as_float(v[q]);
        }
      }
      tcgen05_fence_before();
    }
  }
  if (!ok) atomicExch(&failed, 1u);
  __syncwarp();
  __syncthreads();
  if (failed) {
    if (threadIdx.x == 0) atomicOr(p.status, 1u);
    // copies that were asked for have to land before the CTA gives its memory up
    if (issued > 0) {
      for (unsigned n = issued > S::stages ? issued - S::stages : 0; n < issued; ++n)
        (void)mbarrier_wait(full + 8 * (n % S::stages), (n / S::stages) & 1u, kPolls);
    }
    __syncthreads();
    // a tile that one CTA gives up is given up by its cluster: the others' sums would not be sums of all of k
    for (unsigned i = threadIdx.x; splits > 1 && i < NT * kTileJ; i += kMmaThreads) reinterpret_cast<unsigned*>(stage_mem)[i] = kGivenUp;
  }
  if (splits > 1) {
    __syncwarp();
    cluster.sync();
    // this CTA's columns are split, split + splits, ...: four rows of one column to a thread, all ranks' loads in flight
    const TensorScales ts = tensor_scales(p.a_ts, p.b_ts);
    const unsigned columns = min((unsigned)NT, p.M - i0);
    for (unsigned i = threadIdx.x; split + i / 32 * splits < columns; i += kMmaThreads) {
      const unsigned c = split + i / 32 * splits, row = i % 32 * 4, j = j0 + row;
      float4 v[8];
#pragma unroll
      for (unsigned r = 0; r < 8; ++r)
        if (r < splits) v[r] = *reinterpret_cast<const float4*>(cluster.map_shared_rank(reinterpret_cast<float*>(stage_mem), r) + c * kTileJ + row);
      float4 sum = v[0];
#pragma unroll
      for (unsigned r = 1; r < 8; ++r)
        if (r < splits) sum = make_float4(sum.x + v[r].x, sum.y + v[r].y, sum.z + v[r].z, sum.w + v[r].w);
      if (__builtin_expect(sum.x != sum.x, 0)) {
        bool given_up = false;
        for (unsigned r = 0; r < splits; ++r)
          given_up |= *cluster.map_shared_rank(reinterpret_cast<unsigned*>(stage_mem) + c * kTileJ + row, r) == kGivenUp;
        if (given_up) continue;
      }
      const size_t at = (size_t)(i0 + c) * p.ldo + j;
      T* o = static_cast<T*>(p.out) + at;
      if (j < p.N) o[0] = from_float<T>(sum.x * ts.first * ts.last);
      if (j + 1 < p.N) o[1] = from_float<T>(sum.y * ts.first * ts.last);
      if (j + 2 < p.N) o[2] = from_float<T>(sum.z * ts.first * ts.last);
      if (j + 3 < p.N) o[3] = from_float<T>(sum.w * ts.first * ts.last);
    }
    __syncwarp();
    cluster.sync();                             // nobody leaves while its shared memory is still read
  }
  if (warp == 1) {
    tcgen05_fence_after();
    tmem_free(tmem, S::columns);
  }
}

// ---------------------------------------------------------------------------------------------------------------------
// Many rows on both sides: persistent pairs of CTAs (cta_group::2), each pair a tile of 256 rows of one operand, P (the
// accumulator's lanes), by NT rows of the other, Q (its columns).  A CTA loads 128 rows of P and half of the rows of Q, so an
// operand byte that reaches shared memory serves 256 rows instead of 128, and the bytes from L2 to shared memory are a third
// less than with single CTAs.
//   WIDE           P = A, Q = B: a lane holds neighbours of one row of out; a warp puts 32 rows x 32 columns into shared
//                  memory, and an asynchronous copy takes them out while the warp goes on; for rows of out that start at multiples of
//                  16 bytes and are as many whole 16-byte pieces long: a copy writes all of a piece that it has a part of.
//                  Otherwise P = B, Q = A: the lanes of a warp hold neighbours, stores of one element, coalesced, wherever a row
//                  starts (8192 x 8191 of 8192 columns x 1024 to bf16 nv 48 us instead of 38; the last columns by plain stores
//                  in the same kernel 42, but whole rows then 27.7 instead of 25.6 at 8192 x 8192 x 256)
//   accumulators   two, so that a tile is written out while the next one is multiplied.  Both and the scales' columns do not
//                  fit beside one another at NT = 256: the second starts at `second` < NT, the epilogue drains the shared
//                  columns first and gives the go-ahead after them
//   scales         a set of columns for every stage, or at NT = 256 two in turn: a set is overwritten when the MMAs that
//                  read it are known to be done

template <int FORMAT, int NT, unsigned OUT_BYTES>
struct PairShape {
  static constexpr unsigned blocks = FORMAT == SSGD_MXFP4 ? 2 : 4;
  static constexpr unsigned row_tiles = (NT + 127) / 128;
  static constexpr unsigned p_bytes = 128 * 128, q_bytes = NT / 2 * 128;
  static constexpr unsigned scale_bytes = blocks * 512;
  static constexpr unsigned loaded = p_bytes + q_bytes + (1 + row_tiles) * scale_bytes;     // per CTA and stage
  static constexpr unsigned stage_bytes = (loaded + 1023) / 1024 * 1024;
  static constexpr unsigned box_bytes = 32 * 32 * OUT_BYTES, out_bytes = 8 * box_bytes;   // the eight warps' boxes on their way out
  static constexpr unsigned bar_bytes = 256;
  static constexpr unsigned room_bytes = 232448 - out_bytes - bar_bytes; // for the stages
  static constexpr unsigned stages = room_bytes / stage_bytes < 8 ? room_bytes / stage_bytes : 8;
  static constexpr unsigned scale_columns = (1 + row_tiles) * blocks * 4;
  static constexpr unsigned ring = NT == 256 ? 2 : stages;              // sets of scale columns
  static constexpr unsigned first_scale = 512 - ring * scale_columns;
  static constexpr unsigned room = (first_scale - NT) / 32 * 32;
  static constexpr unsigned second = room < NT ? room : NT;              // column of the second accumulator
  static constexpr unsigned smem = stages * stage_bytes + out_bytes + bar_bytes;      // no other shared memory: the stages start at its base
  static_assert(stages >= 3 && (2 * stages + 3) * 8 + 8 <= bar_bytes, "shared memory");
  static_assert(second + NT <= first_scale && (NT == 256 || second == NT), "tensor memory");
};

struct PairArgs {
  const float* p_ts;
  const float* q_ts;
  void* out;
  unsigned* status;
  size_t ldo;
  unsigned P, Q, k_chunks, tiles_p, tiles_q;    // rows and tiles of either side
  unsigned starve;                              // bytes that a stage waits for in vain: 0 but in the self-test of the waits
};

// Tiles go through bands of eight of P's tiles, so that those in flight share rows of both operands.
struct TilePlace { unsigned p0, q0; };
template <int NT>
__device__ __forceinline__ TilePlace tile_place(unsigned tile, const PairArgs& a) {
  constexpr unsigned kBand = 8;
  const unsigned band = tile / (kBand * a.tiles_q), in = tile - band * kBand * a.tiles_q, high = min(kBand, a.tiles_p - band * kBand);
  return {(band * kBand + in % high) * 256, in / high * NT};
}

template <int FORMAT, int NT, typename T, bool WIDE>
__global__ void __launch_bounds__(kMmaThreads, 1)
fp4_matmul_pair_kernel(const __grid_constant__ CUtensorMap p_map, const __grid_constant__ CUtensorMap q_map,
                       const __grid_constant__ CUtensorMap p_scale_map, const __grid_constant__ CUtensorMap q_scale_map,
                       const __grid_constant__ CUtensorMap out_map, const PairArgs p) {
  using S = PairShape<FORMAT, NT, sizeof(T)>;
  extern __shared__ __align__(1024) unsigned char pair_smem[];           // stages, boxes, barriers; the same place in both CTAs
  uint64_t* bars = reinterpret_cast<uint64_t*>(pair_smem + S::stages * S::stage_bytes + S::out_bytes);
  unsigned &tmem_base = *reinterpret_cast<unsigned*>(bars + 2 * S::stages + 3), &failed = *(&tmem_base + 1);
  const unsigned rank = cluster_rank();
  const unsigned stage0 = smem_u32(pair_smem);
  const unsigned full = smem_u32(bars), empty = full + 8 * S::stages, acc_full = empty + 8 * S::stages, acc_free = acc_full + 8, ended = acc_free + 8;
  const unsigned warp = threadIdx.x >> 5, lane = threadIdx.x & 31u;
  const unsigned stages_k = (p.k_chunks + 3) / 4;
  const unsigned pair = blockIdx.x / 2, pairs = gridDim.x / 2, tiles = p.tiles_p * p.tiles_q;

  if (threadIdx.x == 0) {
    prefetch_tensor_map(&q_map);
    prefetch_tensor_map(&p_map);
    prefetch_tensor_map(&q_scale_map);
    prefetch_tensor_map(&p_scale_map);
    if (WIDE) prefetch_tensor_map(&out_map);
    for (unsigned s = 0; s < S::stages; ++s) {
      mbarrier_init(full + 8 * s, 1);
      mbarrier_init(empty + 8 * s, 1);
    }
    mbarrier_init(acc_full, 1);
    mbarrier_init(ended, 1);
    mbarrier_init(acc_free, 16);                // one arrival from each of the two CTAs' eight epilogue warps
    mbarrier_init_fence();
    failed = 0;
  }
  pdl_launch_dependents();
  pdl_wait();                                   // before tensor memory is taken: its last holder has finished
  if (warp == 1) tmem_alloc_pair(smem_u32(&tmem_base), 512);
  tcgen05_fence_before();
  __syncthreads();
  cluster_sync();                               // the other CTA's barriers are ready too
  tcgen05_fence_after();
  const unsigned tmem = tmem_base;
  bool ok = true;
  unsigned n = 0;                               // stages so far, over all tiles

  if (warp == 0) {
    if (elect_one()) {
      for (unsigned tile = pair; tile < tiles && ok; tile += pairs) {
        const TilePlace at = tile_place<NT>(tile, p);
        const unsigned p0 = at.p0 + rank * 128, q0 = at.q0;
        for (unsigned k = 0; k < stages_k; ++k, ++n) {
          const unsigned s = n % S::stages;
          if (n >= S::stages) ok = mbarrier_wait(empty + 8 * s, (n / S::stages - 1) & 1u, kPolls);
          if (!ok) break;
          const unsigned base = stage0 + s * S::stage_bytes, bar = cluster_address(full + 8 * s, 0);
          if (rank == 0) mbarrier_expect(full + 8 * s, 2 * S::loaded + p.starve);
          tma_load_2d_pair(base, &p_map, (int)(k * 128), (int)p0, bar);
          tma_load_2d_pair(base + S::p_bytes, &q_map, (int)(k * 128), (int)(q0 + rank * (NT / 2)), bar);
          const unsigned sc = base + S::p_bytes + S::q_bytes;
          tma_load_2d_pair(sc, &p_scale_map, (int)(k * S::blocks * 64), (int)(p0 / 128), bar);
          tma_load_2d_pair(sc + S::scale_bytes, &q_scale_map, (int)(k * S::blocks * 64), (int)(q0 / 128), bar);
        }
      }
      // the last stages' commits have to arrive before this CTA may go
      for (unsigned m = n > S::stages ? n - S::stages : 0; m < n && ok; ++m)
        ok = mbarrier_wait(empty + 8 * (m % S::stages), (m / S::stages) & 1u, kPolls);
    }
  } else if (warp == 1) {
    if (rank == 0 && elect_one()) {
      const uint64_t p_desc = smem_descriptor(stage0, 1024, 2), q_desc = smem_descriptor(stage0 + S::p_bytes, 1024, 2),
                     sc_desc = smem_descriptor(stage0 + S::p_bytes + S::q_bytes, 128, 0);
      unsigned s = 0, parity = 0, ring = 0;     // place among the stages and the sets of scale columns
      unsigned behind = 0, behind_parity = 0;   // the stage whose MMAs read the next stage's scale columns last
      bool ready = false, ring_free = true;     // what is known of the next stage's operands and scale columns
      unsigned t = 0;                           // tiles so far
      for (unsigned tile = pair; tile < tiles && ok; tile += pairs, ++t) {
        if (t > 0) ok = mbarrier_wait_cluster(acc_free, (t - 1) & 1u, kPolls);
        if (!ok) break;
        tcgen05_fence_after();
        const unsigned d = tmem + (t & 1u) * S::second;
        const unsigned half = tile_place<NT>(tile, p).q0 % 128 / 32;           // NT = 64: where its rows' scales begin in their tile
        for (unsigned k = 0; k < stages_k; ++k, ++n) {
          ok = (ready || mbarrier_wait(full + 8 * s, parity, kPolls)) && (ring_free || mbarrier_wait(empty + 8 * behind, behind_parity, kPolls));
          if (!ok) break;
          tcgen05_fence_after();
          const unsigned next = s + 1 == S::stages ? 0 : s + 1, next_parity = parity ^ (next == 0);
          ready = mbarrier_test(full + 8 * next, next_parity);    // its answer comes while this stage is issued
          if (S::ring < S::stages && n + 1 >= S::ring) {          // the scale columns of the next stage were last read `ring` stages before it
            if (n + 1 > S::ring) {
              behind_parity ^= behind + 1 == S::stages;
              behind = behind + 1 == S::stages ? 0 : behind + 1;
            }
            ring_free = mbarrier_test(empty + 8 * behind, behind_parity);
          }
          const unsigned at = s * (S::stage_bytes >> 4);
          issue_stage<FORMAT, NT, true>(d, p_desc + at, q_desc + at, sc_desc + at, tmem + S::first_scale + ring * S::scale_columns, half,
                                        p.k_chunks - k * 4, k == 0);
          tcgen05_commit_pair(empty + 8 * s);
          s = next;
          parity = next_parity;
          ring = ring + 1 == S::ring ? 0 : ring + 1;
        }
        if (ok) tcgen05_commit_pair(acc_full);
      }
      if (!ok) {                                // what was issued has to end before tensor memory is freed; nobody writes it out
        tcgen05_commit_pair(ended);
        (void)mbarrier_wait(ended, 0, kPolls);
      }
    }
  } else {
    // Two warps share a quarter of the lanes, units of kUnit columns in turn.
    constexpr unsigned kUnit = 32, kUnits = NT / kUnit, kSharedUnits = (NT - S::second) / kUnit;
    const unsigned quarter = warp & 3u, odd = warp >= 6;
    const TensorScales ts = tensor_scales(p.p_ts, p.q_ts);
    const unsigned go = cluster_address(acc_free, 0), box = stage0 + S::stages * S::stage_bytes + (warp - 2) * S::box_bytes;
    unsigned t = 0;
    for (unsigned tile = pair; tile < tiles; tile += pairs, ++t) {
      ok = mbarrier_wait(acc_full, t & 1u, 4 * kPolls + 64 * stages_k);
      if (!ok) break;
      tcgen05_fence_after();
      const TilePlace at = tile_place<NT>(tile, p);
      const unsigned row0 = at.p0 + rank * 128 + quarter * 32, q0 = at.q0;             // of P; the first of Q
      const unsigned lanes = tmem + (t & 1u) * S::second + (quarter << 21);
      // the columns that both accumulators use come first: from `second` on in the first, the front ones in the second
      const unsigned first = (t & 1u) ? 0u : S::second % NT;
      if (odd + 1 > kSharedUnits && lane == 0) mbarrier_arrive_cluster(go);            // none of them is this warp's
#pragma unroll 1
      for (unsigned unit = odd; unit < kUnits; unit += 2) {
        const unsigned c = (first + unit * kUnit) % NT;
        unsigned v[32];
        tmem_read32(lanes + c, v);
        if (kSharedUnits > 0 && unit + 1 <= kSharedUnits && unit + 2 >= kSharedUnits) {                       // this warp's last shared columns
          tcgen05_fence_before();
          __syncwarp();
          if (lane == 0) mbarrier_arrive_cluster(go);
        }
        if (row0 < p.P && q0 + c < p.Q) {
          scale_first(v, ts);
          if constexpr (WIDE) {
            if (lane == 0) tma_store_wait_read();                                      // the box is free again
            __syncwarp();
            if constexpr (sizeof(T) == 2) {                                            // rows of 64 bytes, 64-byte swizzle
#pragma unroll
              for (unsigned q = 0; q < 16; ++q) v[q] = pack2(T(), __uint_as_float(v[2 * q]) * ts.last, __uint_as_float(v[2 * q + 1]) * ts.last);
#pragma unroll
              for (unsigned q = 0; q < 4; ++q)
                store_shared16(box + lane * 64 + ((q ^ (lane >> 1 & 3u)) << 4), v[4 * q], v[4 * q + 1], v[4 * q + 2], v[4 * q + 3]);
            } else {                                                                   // rows of 128 bytes, 128-byte swizzle
#pragma unroll
              for (unsigned q = 0; q < 32; ++q) v[q] = __float_as_uint(__uint_as_float(v[q]) * ts.last);
#pragma unroll
              for (unsigned q = 0; q < 8; ++q)
                store_shared16(box + lane * 128 + ((q ^ (lane & 7u)) << 4), v[4 * q], v[4 * q + 1], v[4 * q + 2], v[4 * q + 3]);
            }
            async_proxy_fence();
            __syncwarp();
            if (lane == 0) tma_store_2d(&out_map, (int)(q0 + c), (int)row0, box);
          } else if (row0 + lane < p.P) {
            store_column(static_cast<T*>(p.out) + (size_t)(q0 + c) * p.ldo + row0 + lane, p.ldo, v, min(32u, p.Q - (q0 + c)), ts.last);
          }
        }
        __syncwarp();
      }
      tcgen05_fence_before();
    }
    if (WIDE && lane == 0) tma_store_wait();
  }
  if (!ok) atomicExch(&failed, 1u);
  __syncwarp();
  __syncthreads();
  if (failed) {
    // copies that were asked for, here and by the other CTA, have to land before the memory is given up
    if (threadIdx.x == 0) atomicOr(p.status, 1u);
    if (rank == 0 && warp == 0)
      for (unsigned m = n > S::stages ? n - S::stages : 0; m < n; ++m)
        (void)mbarrier_wait(full + 8 * (m % S::stages), (m / S::stages) & 1u, kPolls);
  }
  __syncthreads();
  cluster_sync();
  if (warp == 1) {
    tcgen05_fence_after();
    tmem_free_pair(tmem, 512);
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

// Scale tiles as a matrix of 64-bit words, a tile of 512 bytes 64 of them, in boxes of box_tiles x box_rows tiles.
bool scale_map(CUtensorMap* map, const uint8_t* scales, size_t row_tiles, size_t tiles_k, unsigned box_tiles, unsigned box_rows) {
  const EncodeTiled f = encode_tiled();
  if (!f) return false;
  const cuuint64_t dims[2] = {tiles_k * 64, row_tiles}, strides[1] = {tiles_k * 512};
  const cuuint32_t box[2] = {box_tiles * 64, box_rows}, steps[2] = {1, 1};
  return f(map, CU_TENSOR_MAP_DATA_TYPE_UINT64, 2, const_cast<uint8_t*>(scales), dims, strides, box, steps, CU_TENSOR_MAP_INTERLEAVE_NONE,
           CU_TENSOR_MAP_SWIZZLE_NONE, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// out as boxes of 32 columns x 32 rows, swizzled over the 64 or 128 bytes of a row; cols in whole 16-byte pieces.
bool out_map_of(CUtensorMap* map, void* out, int dtype, size_t rows, size_t cols, size_t ldo) {
  const EncodeTiled f = encode_tiled();
  if (!f) return false;
  const size_t e = dtype_bytes((unsigned)dtype);
  const cuuint64_t dims[2] = {cols, rows}, strides[1] = {ldo * e};
  const cuuint32_t box[2] = {32, 32}, steps[2] = {1, 1};
  return f(map, dtype == SSGD_F32 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT32 : dtype == SSGD_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16,
           2, out, dims, strides, box, steps, CU_TENSOR_MAP_INTERLEAVE_NONE, e == 4 ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_64B, CU_TENSOR_MAP_L2_PROMOTION_NONE,
           CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <int FORMAT, int NT, typename T>
ssgd_status launch_product(const CUtensorMap& a_map, const CUtensorMap& b_map, const ProductArgs& p, unsigned tiles, unsigned splits, cudaStream_t s) {
  using S = Shape<FORMAT, NT>;
  auto kernel = fp4_matmul_kernel<FORMAT, NT, T>;
  static unsigned long long seen = 0;
  if (!allow_smem(reinterpret_cast<const void*>(kernel), S::smem, &seen)) return SSGD_ERR_CUDA;
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

struct Operands {
  const uint8_t *a, *a_scales, *b, *b_scales;
  const float *a_ts, *b_ts;
  size_t M, N, K;
  void* out;
  int dtype;
  size_t ldo;
  unsigned* status;
  unsigned starve;
};

template <int FORMAT, int NT>
ssgd_status launch_product_typed(const CUtensorMap& a_map, const CUtensorMap& b_map, const ProductArgs& p, int dtype, unsigned tiles, unsigned splits,
                                 cudaStream_t s) {
  switch (dtype) {
    case SSGD_F32: return launch_product<FORMAT, NT, float>(a_map, b_map, p, tiles, splits, s);
    case SSGD_BF16: return launch_product<FORMAT, NT, __nv_bfloat16>(a_map, b_map, p, tiles, splits, s);
    default: return launch_product<FORMAT, NT, __half>(a_map, b_map, p, tiles, splits, s);
  }
}

// CTAs that share one tile's k.  A stage costs 0.12 to 0.2 us, joining the parts about 1 us (B200; one row against 4096 x K,
// one / two / four CTAs: 3.6 / 4.4 / 4.6 us at K = 1024, 5.9 / 5.6 / 5.5 at 4096, 9.5 / 7.8 / 7.3 at 8192).  Clusters have to
// find their place at the same time: four CTAs fit 32 times, eight 12 times; one tile more doubles the time.
inline unsigned k_splits(unsigned tiles, unsigned stages_k, int sms) {
  if (stages_k >= 16 && tiles * 12 <= (unsigned)sms) return 8;
  if (stages_k >= 12 && tiles * 37 <= (unsigned)sms * 8) return 4;
  if (stages_k >= 14 && tiles * 2 <= (unsigned)sms) return 2;
  return 1;
}

// The form of a product: by single CTAs, tiles of 128 rows of B by nt rows of A, k split over `splits` of them; or by pairs, tiles of
// 256 x nt, WIDE where rows of out allow it.
struct Form {
  bool pairs, wide;
  unsigned nt, splits;
  size_t tiles;
};
Form choose_form(size_t M, size_t N, size_t K, bool rows_of_16_bytes, int sms);

template <int FORMAT>
ssgd_status product(const Operands& o, const Form& form, cudaStream_t s) {
  const size_t row_bytes = ssgd_fp4_row_bytes(o.K);
  const unsigned nt = form.nt, splits = form.splits;
  const size_t tiles_i = (o.M + nt - 1) / nt;
  if (form.tiles > (size_t)1 << 27) return SSGD_ERR_SIZE;
  const unsigned tiles = (unsigned)form.tiles;
  CUtensorMap a_map, b_map;
  if (!code_map(&a_map, o.a, o.M, row_bytes, nt) || !code_map(&b_map, o.b, o.N, row_bytes, kTileJ)) return SSGD_ERR_CUDA;
  ProductArgs p;
  p.a_scales = o.a_scales; p.b_scales = o.b_scales; p.a_ts = o.a_ts; p.b_ts = o.b_ts; p.out = o.out; p.status = o.status; p.ldo = o.ldo;
  p.M = (unsigned)o.M; p.N = (unsigned)o.N;
  p.k_chunks = (unsigned)((row_bytes + 31) / 32);
  p.tiles_k = (unsigned)((fp4_block_count(FORMAT, o.K) + 3) / 4);
  p.tiles_i = (unsigned)tiles_i;
  p.starve = o.starve;
  switch (nt) {
    case 16: return launch_product_typed<FORMAT, 16>(a_map, b_map, p, o.dtype, tiles, splits, s);
    case 32: return launch_product_typed<FORMAT, 32>(a_map, b_map, p, o.dtype, tiles, splits, s);
    case 64: return launch_product_typed<FORMAT, 64>(a_map, b_map, p, o.dtype, tiles, splits, s);
    default: return launch_product_typed<FORMAT, 128>(a_map, b_map, p, o.dtype, tiles, splits, s);
  }
}

template <int FORMAT, int NT, typename T, bool WIDE>
ssgd_status launch_pair(const Operands& o, int sms, cudaStream_t s) {
  using S = PairShape<FORMAT, NT, sizeof(T)>;
  const size_t row_bytes = ssgd_fp4_row_bytes(o.K), tiles_k = (fp4_block_count(FORMAT, o.K) + 3) / 4;
  const size_t P = WIDE ? o.M : o.N, Q = WIDE ? o.N : o.M, tiles_p = (P + 255) / 256, tiles_q = (Q + NT - 1) / NT;
  if (tiles_p * tiles_q > kMaxGrid / 8) return SSGD_ERR_SIZE;
  CUtensorMap p_map, q_map, p_scale_map, q_scale_map, out_map;
  if (!code_map(&p_map, WIDE ? o.a : o.b, P, row_bytes, 128) || !code_map(&q_map, WIDE ? o.b : o.a, Q, row_bytes, NT / 2) ||
      !scale_map(&p_scale_map, WIDE ? o.a_scales : o.b_scales, (P + 127) / 128, tiles_k, S::blocks, 1) ||
      !scale_map(&q_scale_map, WIDE ? o.b_scales : o.a_scales, (Q + 127) / 128, tiles_k, S::blocks, S::row_tiles))
    return SSGD_ERR_CUDA;
  if (!WIDE) out_map = p_map;                    // not used
  else if (!out_map_of(&out_map, o.out, o.dtype, o.M, o.N, o.ldo)) return SSGD_ERR_CUDA;
  PairArgs p;
  p.p_ts = o.a_ts; p.q_ts = o.b_ts; p.out = o.out; p.status = o.status; p.ldo = o.ldo;
  p.P = (unsigned)P; p.Q = (unsigned)Q;
  p.k_chunks = (unsigned)((row_bytes + 31) / 32);
  p.tiles_p = (unsigned)tiles_p;
  p.tiles_q = (unsigned)tiles_q;
  p.starve = o.starve;
  auto kernel = fp4_matmul_pair_kernel<FORMAT, NT, T, WIDE>;
  static unsigned long long seen = 0;
  if (!allow_smem(reinterpret_cast<const void*>(kernel), S::smem, &seen)) return SSGD_ERR_CUDA;
  const size_t tiles = tiles_p * tiles_q;
  const unsigned pairs = (unsigned)(tiles < (size_t)(sms / 2) ? tiles : (size_t)(sms / 2));
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(2 * pairs);
  cfg.blockDim = dim3(kMmaThreads);
  cfg.dynamicSmemBytes = S::smem;
  cfg.stream = s;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = 2;
  attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 2;
  (void)cudaLaunchKernelEx(&cfg, kernel, p_map, q_map, p_scale_map, q_scale_map, out_map, p);
  return launch_status();
}

template <int FORMAT, int NT, typename T>
ssgd_status pair_typed(const Operands& o, bool wide, int sms, cudaStream_t s) {
  return wide ? launch_pair<FORMAT, NT, T, true>(o, sms, s) : launch_pair<FORMAT, NT, T, false>(o, sms, s);
}

template <int FORMAT, int NT>
ssgd_status pair_product(const Operands& o, bool wide, int sms, cudaStream_t s) {
  switch (o.dtype) {
    case SSGD_F32: return pair_typed<FORMAT, NT, float>(o, wide, sms, s);
    case SSGD_BF16: return pair_typed<FORMAT, NT, __nv_bfloat16>(o, wide, sms, s);
    default: return pair_typed<FORMAT, NT, __half>(o, wide, sms, s);
  }
}

// Nanoseconds of a product by pairs with tiles of 256 x nt, fitted on B200: a start, a stage, and for each further tile of a
// pair its stages or its writing out, whichever is longer.  Measured, nt = 64 / 128 / 256 in us: 2048 x 1024 x 4096 10.2 / 7.9 /
// 10.7; 2048 x 4096 x 1024 12.3 / 9.2 / 9.3; 777 x 1111 x 1500 5.8 / 6.4 / 8.5; 8192 x 8192 x 256 46 / 28 / 25.  Over 22 shapes in
// two types the choice was within 5 % of the best of the three but for two (10 and 11 %).
inline unsigned long long pair_cost(unsigned long long tiles_p, size_t Q, unsigned nt, unsigned long long stages_k, unsigned pairs) {
  const unsigned long long tiles = tiles_p * ((Q + nt - 1) / nt), rounds = (tiles + pairs - 1) / pairs;
  const unsigned start = nt == 64 ? 3900 : nt == 128 ? 4400 : 5600, stage = nt == 64 ? 123 : nt == 128 ? 160 : 300,
                 write = nt == 64 ? 1000 : nt == 128 ? 1350 : 2100;
  const unsigned long long work = stages_k * stage;
  return start + work + (rounds - 1) * (work + 250 > write ? work + 250 : write);
}

Form choose_form(size_t M, size_t N, size_t K, bool rows_of_16_bytes, int sms) {
  // Up to 128 rows of A: the weight's rows are the lanes and stream through once.  More rows, but few tiles and a long k: the
  // same kernel, because it splits k (150 x 300 x 16384: 8.5 us against 13.8 by pairs; x 4096 7.3 against 6.7).
  const size_t stages_k = (ssgd_fp4_row_bytes(K) + 127) / 128, tiles_j = (N + kTileJ - 1) / kTileJ;
  if (M <= 128 || (stages_k >= 24 && ((M + 127) / 128) * tiles_j * 8 <= (size_t)sms)) {
    const unsigned nt = M <= 16 ? 16 : M <= 32 ? 32 : M <= 64 ? 64 : 128;
    const size_t tiles = tiles_j * ((M + nt - 1) / nt);
    return {false, false, nt, k_splits((unsigned)tiles, (unsigned)stages_k, sms), tiles};
  }
  const bool wide = rows_of_16_bytes;
  const size_t P = wide ? M : N, Q = wide ? N : M, tiles_p = (P + 255) / 256;
  const unsigned pairs = (unsigned)(sms / 2);
  const unsigned long long c64 = pair_cost(tiles_p, Q, 64, stages_k, pairs), c128 = pair_cost(tiles_p, Q, 128, stages_k, pairs),
                           c256 = pair_cost(tiles_p, Q, 256, stages_k, pairs);
  const unsigned nt = c256 <= c128 && c256 <= c64 ? 256 : c128 <= c64 ? 128 : 64;
  return {true, wide, nt, 1, tiles_p * ((Q + nt - 1) / nt)};
}

// Rows of out in whole 16-byte pieces, at a stride that a tensor map holds.
inline bool rows_of_16_bytes(const void* out, size_t N, size_t ldo, int dtype) {
  const size_t e = dtype_bytes((unsigned)dtype);
  return aligned16(out) && ldo * e % 16 == 0 && N * e % 16 == 0 && ldo < (size_t)1 << 37;
}

template <int FORMAT>
ssgd_status any_product(const Operands& o, int sms, cudaStream_t s) {
  const Form form = choose_form(o.M, o.N, o.K, rows_of_16_bytes(o.out, o.N, o.ldo, o.dtype), sms);
  if (!form.pairs) return product<FORMAT>(o, form, s);
  return form.nt == 256   ? pair_product<FORMAT, 256>(o, form.wide, sms, s)
         : form.nt == 128 ? pair_product<FORMAT, 128>(o, form.wide, sms, s)
                          : pair_product<FORMAT, 64>(o, form.wide, sms, s);
}

ssgd_status checked_product(const uint8_t* a_codes, const uint8_t* a_scales, const float* a_tensor_scale, const uint8_t* b_codes, const uint8_t* b_scales,
                            const float* b_tensor_scale, size_t M, size_t N, size_t K, int format, void* out, int dtype, size_t ldo, unsigned* status,
                            unsigned starve, void* stream) {
  if (!fp4_format_ok(format) || dtype_bytes((unsigned)dtype) == 0) return SSGD_ERR_ARG;
  if (!a_codes || !a_scales || !b_codes || !b_scales || !out || !status) return SSGD_ERR_NULL;
  if (M > SSGD_FP4_MAX_SIDE || N > SSGD_FP4_MAX_SIDE || K > SSGD_FP4_MAX_SIDE || ldo < N || mul_overflows(M, ldo) || mul_overflows(M * ldo, 4))
    return SSGD_ERR_SIZE;
  if (!aligned16(a_codes) || !aligned16(a_scales) || !aligned16(b_codes) || !aligned16(b_scales) ||
      reinterpret_cast<uintptr_t>(out) % dtype_bytes((unsigned)dtype) != 0 ||
      ((reinterpret_cast<uintptr_t>(a_tensor_scale) | reinterpret_cast<uintptr_t>(b_tensor_scale) | reinterpret_cast<uintptr_t>(status)) & 3u))
    return SSGD_ERR_ALIGN;
  if (format == SSGD_MXFP4 && (a_tensor_scale || b_tensor_scale)) return SSGD_ERR_ARG;
  if (M == 0 || N == 0) return SSGD_OK;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  if (K == 0) {
    const size_t e = dtype_bytes((unsigned)dtype);
    return cudaMemset2DAsync(out, ldo * e, 0, N * e, M, s) == cudaSuccess ? SSGD_OK : SSGD_ERR_CUDA;
  }
  DeviceInfo info;
  if (!device_info(&info)) return SSGD_ERR_CUDA;
  const Operands o = {a_codes, a_scales, b_codes, b_scales, a_tensor_scale, b_tensor_scale, M, N, K, out, dtype, ldo, status, starve};
  return format == SSGD_MXFP4 ? any_product<SSGD_MXFP4>(o, info.sms, s) : any_product<SSGD_NVFP4>(o, info.sms, s);
}

}  // namespace

extern "C" {

ssgd_status ssgd_fp4_matmul(const uint8_t* a_codes, const uint8_t* a_scales, const float* a_tensor_scale, const uint8_t* b_codes,
                            const uint8_t* b_scales, const float* b_tensor_scale, size_t M, size_t N, size_t K, int format, void* out,
                            int dtype, size_t ldo, unsigned* status, void* stream) {
  return checked_product(a_codes, a_scales, a_tensor_scale, b_codes, b_scales, b_tensor_scale, M, N, K, format, out, dtype, ldo, status, 0, stream);
}

ssgd_status ssgd_fp4_matmul_form(size_t M, size_t N, size_t K, int dtype, size_t ldo, int sms, unsigned* form) {
  if (!form) return SSGD_ERR_NULL;
  if (dtype_bytes((unsigned)dtype) == 0 || sms < 2) return SSGD_ERR_ARG;
  if (M < 1 || N < 1 || K < 1 || M > SSGD_FP4_MAX_SIDE || N > SSGD_FP4_MAX_SIDE || K > SSGD_FP4_MAX_SIDE || ldo < N) return SSGD_ERR_SIZE;
  const Form f = choose_form(M, N, K, rows_of_16_bytes(nullptr, N, ldo, dtype), sms);
  const size_t most = f.pairs ? (size_t)(sms / 2) : f.tiles;
  form[0] = f.pairs ? 2 : 1;
  form[1] = f.nt;
  form[2] = f.splits;
  form[3] = f.wide;
  form[4] = (unsigned)((f.tiles + most - 1) / most);
  return SSGD_OK;
}

ssgd_status ssgd_fp4_matmul_wait_selftest(const uint8_t* a_codes, const uint8_t* a_scales, const uint8_t* b_codes, const uint8_t* b_scales, size_t M,
                                          size_t N, size_t K, int format, void* out, int dtype, size_t ldo, unsigned* status, void* stream) {
  // one tile of a pair, two stages, or a few tiles whose k may be split: the waits run out once
  if (M > 256 || N > 256 || K > (M <= 128 ? 4096 : 512)) return SSGD_ERR_SIZE;
  return checked_product(a_codes, a_scales, nullptr, b_codes, b_scales, nullptr, M, N, K, format, out, dtype, ldo, status, 16, stream);
}

ssgd_status ssgd_fp4_matmul_block(const uint64_t* a) {
  if (!a) return SSGD_ERR_NULL;
  return ssgd_fp4_matmul(block_ptr<const uint8_t>(a[0]), block_ptr<const uint8_t>(a[1]), block_ptr<const float>(a[2]), block_ptr<const uint8_t>(a[3]),
                         block_ptr<const uint8_t>(a[4]), block_ptr<const float>(a[5]), a[6], a[7], a[8], (int)a[9], block_ptr<void>(a[10]), (int)a[11],
                         a[12], block_ptr<unsigned>(a[13]), block_ptr<void>(a[14]));
}

}  // extern "C"
