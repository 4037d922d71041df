// Products of 16-bit operands on the tensor cores, out[i][j] = sum_k P[i][k] Q[j][k] in fp32, with what becomes of the sums left to
// the caller: a class that takes 32 neighbouring columns of one row at a time (an epilogue).
//
// A persistent CTA, or pair of CTAs (cta_group::2), takes tiles of 128 (256) rows of P by NT rows of Q in turn.  P's rows are the
// accumulator's lanes, so a thread of the epilogue has neighbours of one row, and what is summed along a row (a softmax)
// needs no exchange between threads.
//   warp 0      one thread brings stages of 64 of k (tiled copies, 128-byte swizzle, zeros beyond the edges)
//   warp 1      one thread issues the MMAs, four of 16 of k a stage
//   warps 4..11 read the accumulators, two warps to a quarter of the lanes, 32 columns in turn; two accumulators, so that a tile
//               is written out while the next is multiplied
// An operand may lie in memory with its k side by side, or with its rows side by side (a matrix that another product
// takes the other way round): the copies and the tensor cores take both, nothing is transposed.
// TERMS = 3: each operand is a sum of two fp16 matrices, high and low part (22 bits together); high * low, low * high and high * high
// go into the same sum, the small ones first; low * low is below the last bit that counts.
// CHUNK > 0: the tensor cores add with fp32 accumulators, but cut off what does not fit instead of rounding it, so that a sum is off
// by up to 2^-24 of itself for each 16 of k, always to the same side (measured: 10^-8 of the sum for each of k).  Where that
// counts the sum is taken every CHUNK stages, and the parts are added by the epilogue's threads, rounded to nearest.
// Every wait has an iteration limit and reports through a status word, as in the 4-bit product.
#ifndef SSGD_HALF_PRODUCT_CUH_
#define SSGD_HALF_PRODUCT_CUH_

#include <type_traits>

#include "host_calls.h"
#include "dtypes.cuh"
#include "sm100.cuh"
#include "tensor_map.h"

namespace {

constexpr int kHalfThreads = 384;                 // a warpgroup for copies and MMAs, two that write out
constexpr unsigned kHalfPolls = 200000;           // bound of a wait, about 0.2 s

// ---------------------------------------------------------------------------------------------------------------------
// What epilogues share.  A thread has 32 neighbours of a row, memory wants neighbours from the lanes of a warp: 32 x 32 elements
// change hands in a warp's box.  (Threads that went to memory by themselves, 16 bytes of their rows at a time, made 32 lookups of every
// access: 480 us for 24 matrices of 1024 x 4096 where their product takes 150.)

// Two numbers as the sum of two fp16 numbers each, 22 bits together.
__device__ __forceinline__ void split_pair(float a, float b, unsigned& high, unsigned& low) {
  high = pack2(__half(), a, b);
  low = pack2(__half(), a - low_to_float(__half(), high), b - high_to_float(__half(), high));
}
__device__ __forceinline__ void store_shared2(unsigned at, unsigned v) {
  asm volatile("st.shared.b16 [%0], %1;" ::"r"(at), "h"((unsigned short)v) : "memory");
}

struct Box {
  unsigned at, full, lane;      // shared memory; two barriers; this thread
  bool fine = true;             // no wait has run out
  unsigned pending = 0, phase = 0;      // bits of the two barriers: asked for and not yet there; parity
  __device__ __forceinline__ Box(unsigned at_, unsigned full_, unsigned lane_) : at(at_), full(full_), lane(lane_) {}

  // 16-bit elements, a row 64 bytes, as copies with 64-byte swizzle have them.
  __device__ __forceinline__ unsigned place16(unsigned offset, unsigned row, unsigned piece) const {
    return at + offset + row * 64 + ((piece ^ (row >> 1 & 3u)) << 4);
  }
  template <typename T>
  __device__ __forceinline__ void put16(unsigned offset, const float* v) const {
#pragma unroll
    for (unsigned q = 0; q < 4; ++q)
      store_shared16(place16(offset, lane, q), pack2(T(), v[8 * q], v[8 * q + 1]), pack2(T(), v[8 * q + 2], v[8 * q + 3]), pack2(T(), v[8 * q + 4], v[8 * q + 5]),
                     pack2(T(), v[8 * q + 6], v[8 * q + 7]));
  }
  // 32 elements of 16 bits, in words: this thread's row, or, transposed, a column of the box.
  __device__ __forceinline__ void put_words(unsigned offset, const unsigned (&w)[16]) const {
#pragma unroll
    for (unsigned q = 0; q < 4; ++q) store_shared16(place16(offset, lane, q), w[4 * q], w[4 * q + 1], w[4 * q + 2], w[4 * q + 3]);
  }
  __device__ __forceinline__ void put_words_across(unsigned offset, const unsigned (&w)[16]) const {
#pragma unroll
    for (unsigned q = 0; q < 16; ++q) {
      store_shared2(place16(offset, 2 * q, lane >> 3) + (lane & 7u) * 2, w[q]);
      store_shared2(place16(offset, 2 * q + 1, lane >> 3) + (lane & 7u) * 2, w[q] >> 16);
    }
  }
  __device__ __forceinline__ void get8(unsigned offset, unsigned piece, float (&v)[8]) const {
    unsigned a, b, c, d;
    asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(a), "=r"(b), "=r"(c), "=r"(d) : "r"(place16(offset, lane, piece)) : "memory");
    v[0] = low_to_float(__half(), a); v[1] = high_to_float(__half(), a); v[2] = low_to_float(__half(), b); v[3] = high_to_float(__half(), b);
    v[4] = low_to_float(__half(), c); v[5] = high_to_float(__half(), c); v[6] = low_to_float(__half(), d); v[7] = high_to_float(__half(), d);
  }
  // Shared memory as the threads have written it goes out; several may follow one another behind one fence.
  __device__ __forceinline__ void fence() const {
    async_proxy_fence();
    __syncwarp();
  }
  __device__ __forceinline__ void send(const CUtensorMap& map, unsigned offset, unsigned x, unsigned y, unsigned z) const {
    if (lane == 0) tma_store_3d(&map, (int)x, (int)y, (int)z, at + offset);
  }
  // What went out may be overwritten.
  __device__ __forceinline__ void sent() const {
    if (lane == 0) tma_store_wait_read();
    __syncwarp();
  }
  __device__ __forceinline__ void sent_but_last() const {
    if (lane == 0) tma_store_wait_read_but_last();
    __syncwarp();
  }
  // 32 x 32 elements of 16 bits of one or two matrices to `offset` (and 2048 behind), counted on barrier b; and the wait for them.
  __device__ __forceinline__ void ask(unsigned b, unsigned offset, const CUtensorMap& first, const CUtensorMap* second, unsigned x, unsigned y, unsigned z) {
    if (lane == 0) {
      mbarrier_expect(full + 8 * b, second ? 4096 : 2048);
      tma_load_3d(at + offset, &first, (int)x, (int)y, (int)z, full + 8 * b);
      if (second) tma_load_3d(at + offset + 2048, second, (int)x, (int)y, (int)z, full + 8 * b);
    }
    pending |= 1u << b;
  }
  __device__ __forceinline__ void take(unsigned b) {
    fine = __all_sync(0xFFFFFFFFu, mbarrier_wait(full + 8 * b, phase >> b & 1u, kHalfPolls)) && fine;
    phase ^= 1u << b;
    pending &= ~(1u << b);
  }
  __device__ __forceinline__ void finish() {
    if (lane == 0) tma_store_wait();
    for (unsigned b = 0; b < 2; ++b)
      if (pending >> b & 1u) take(b);           // asked for, and given up before it was used
  }

  // fp32 elements, a row 128 bytes, its eight pieces of 16 in an order of its own, so that rows and columns are read without conflicts.
  __device__ __forceinline__ unsigned place32(unsigned row, unsigned column) const { return at + row * 128 + (((column >> 2) ^ (row & 7u)) << 4) + (column & 3u) * 4; }
  __device__ __forceinline__ void put32(const float* v) const {
    __syncwarp();
#pragma unroll
    for (unsigned q = 0; q < 8; ++q)
      store_shared16(place32(lane, 4 * q), __float_as_uint(v[4 * q]), __float_as_uint(v[4 * q + 1]), __float_as_uint(v[4 * q + 2]), __float_as_uint(v[4 * q + 3]));
    __syncwarp();
  }
  __device__ __forceinline__ float get32(unsigned row, unsigned column) const {
    float v;
    asm volatile("ld.shared.f32 %0, [%1];" : "=f"(v) : "r"(place32(row, column)) : "memory");
    return v;
  }
  // The box's first `rows` rows and `left` columns to memory at any place and stride, lanes side by side: one element each, or, 16 bits
  // that start at multiples of four bytes, two elements of two rows at a time.
  template <typename T>
  __device__ __forceinline__ void rows_out(T* o, size_t ld, unsigned rows, unsigned left, const float* v) const {
    put32(v);
    if (sizeof(T) == 2 && ((reinterpret_cast<uintptr_t>(o) & 3u) | (ld & 1u)) == 0) {
      const unsigned c = (lane & 15u) * 2;
      T* p = o + (lane >> 4) * ld + c;
#pragma unroll 8
      for (unsigned r = lane >> 4; r < rows; r += 2, p += 2 * ld) {
        float a, b;
        asm volatile("ld.shared.v2.f32 {%0, %1}, [%2];" : "=f"(a), "=f"(b) : "r"(place32(r, c)) : "memory");
        if constexpr (sizeof(T) == 2) {
          if (c + 1 < left) *reinterpret_cast<unsigned*>(p) = pack2(T(), a, b);
          else if (c < left) *p = from_float<T>(a);
        }
      }
    } else if (lane < left) {
      T* p = o + lane;
#pragma unroll 8
      for (unsigned r = 0; r < rows; ++r, p += ld) *p = from_float<T>(get32(r, lane));
    }
  }
  // out = f(what is in memory, the box's value), row by row, eight loads in flight.
  template <typename T, typename F>
  __device__ __forceinline__ void rows_join(const float* in, size_t ld_in, T* o, size_t ld, unsigned rows, unsigned left, const float* v, F f) const {
    put32(v);
    if (lane >= left) return;
    for (unsigned r0 = 0; r0 < rows; r0 += 8) {
      float old[8];
#pragma unroll
      for (unsigned u = 0; u < 8; ++u) old[u] = r0 + u < rows ? in[(r0 + u) * ld_in + lane] : 0.0f;
#pragma unroll
      for (unsigned u = 0; u < 8; ++u)
        if (r0 + u < rows) o[(r0 + u) * ld + lane] = from_float<T>(f(old[u], get32(r0 + u, lane)));
    }
  }
};

struct HalfMaps {
  CUtensorMap p[2], q[2];                         // high and low part (TERMS = 3); TERMS = 1: q[1] may be another choice for q
};

struct HalfPlan {
  unsigned P, Q;                                  // rows of the operands of one matrix
  unsigned k_stages, k_chunks;                    // k in pieces of 64 and of 16
  unsigned tiles_p, tiles_q, per_matrix, tiles;   // tiles: per matrix, and of all matrices and splits
  unsigned splits;                                // pieces of k that are summed apart
  unsigned p_box;                                 // rows of P that a CTA loads: fewer than 128 where P has fewer
  unsigned idesc;
  unsigned symmetric;                             // only tiles that reach the diagonal or lie above it
  unsigned starve;                                // bytes that a stage waits for in vain: 0 but in the self-test of the waits
  const unsigned* q_choice;                       // not null: where it points to non-zero, q[1] is taken for q[0]
  unsigned* status;
};

struct HalfPlace { unsigned matrix, split, p0, q0, tile, tile_q, rows; };      // rows: of P in a tile

template <bool PAIR, int NT, int TERMS, int CHUNK, unsigned BOX>
struct HalfShape {
  static constexpr unsigned rows = PAIR ? 256 : 128;                       // of P in a tile
  static constexpr unsigned q_rows = PAIR ? NT / 2 : NT;                   // of Q that a CTA loads
  static constexpr unsigned parts = TERMS == 3 ? 2 : 1;
  static constexpr unsigned p_bytes = 128 * 128, q_bytes = q_rows * 128;
  static constexpr unsigned stage_bytes = parts * (p_bytes + q_bytes);
  static constexpr unsigned box_bytes = BOX, out_bytes = 8 * box_bytes;    // the eight warps' room on the way out
  static constexpr unsigned bar_bytes = 512;
  static constexpr unsigned room = 232448 - out_bytes - bar_bytes;
  static constexpr unsigned stages = room / stage_bytes < 8 ? room / stage_bytes : 8;
  // Accumulators.  Sums that are taken every few stages need several on their way between the tensor cores and the threads: a
  // round takes about 1000 clocks, a stage of 64 columns 128 (TERMS = 1)
  static constexpr unsigned accs = CHUNK > 0 ? 512 / NT : 2, columns = accs * NT;
  // more than half of an SM's shared memory always: CTAs that hold and wait for tensor memory on one SM would never end
  static constexpr unsigned needed = stages * stage_bytes + out_bytes + bar_bytes;
  static constexpr unsigned smem = needed < 118784 ? 118784 : needed;
  static_assert(stages >= 3 && (2 * stages + 1 + 16 + 2 * accs) * 8 + 8 <= bar_bytes && columns <= 512 && q_rows % 64 == 0, "shape");
};

// Tiles go through bands of eight of P's tiles, so that those in flight share rows of both operands.
template <bool PAIR, int NT, bool SPLIT>
__device__ __forceinline__ HalfPlace half_place(unsigned tile, const HalfPlan& p) {
  constexpr unsigned rows = PAIR ? 256 : 128, kBand = 8;
  const unsigned z = tile / p.per_matrix, in_matrix = tile - z * p.per_matrix;
  HalfPlace at;
  at.matrix = !SPLIT && p.splits > 1 ? z / p.splits : z;
  at.split = SPLIT ? 0 : z - at.matrix * p.splits;
  at.tile = in_matrix;
  if (p.symmetric) {
    unsigned i = 0, left = in_matrix;
    while (left >= p.tiles_q - i * (rows / NT)) left -= p.tiles_q - i++ * (rows / NT);
    at.p0 = i * rows;
    at.q0 = (i * (rows / NT) + left) * NT;
  } else {
    const unsigned band = in_matrix / (kBand * p.tiles_q), in = in_matrix - band * kBand * p.tiles_q, high = min(kBand, p.tiles_p - band * kBand);
    at.p0 = (band * kBand + in % high) * rows;
    at.q0 = in / high * NT;
  }
  at.tile_q = at.q0 / NT;
  at.rows = rows;
  return at;
}

// What an epilogue offers, besides its Args:
//   kBox                            bytes of shared memory of a warp
//   prefetch(args)                  of its tensor maps, by one thread
//   begin(args, place, row0, odd)   before a tile's first columns; a thread's row is row0 + lane, odd: which half of the columns
//   ahead(args, column)             before the sums of those columns are there: what it needs of memory may be asked for
//   unit(args, column, left, v)     32 sums of columns column .., `left` of them inside; it may change them
//   end(args, place, warp)          behind the last
//   finish(args)                    behind the last tile
// All threads of a warp call each of them.
// How the operands lie in memory: which of them with their rows side by side.
enum HalfLayout { kBothByK = 0, kQByRows = 1, kBothByRows = 3 };

// One stage's MMAs, with descriptors that differ by constants: what the issuing thread computes between two of them the tensor cores may
// have to wait for.
template <bool PAIR, int TERMS, int LAYOUT, unsigned LOW>
__device__ __forceinline__ void half_issue(unsigned d, uint64_t pd, uint64_t qd, unsigned idesc, unsigned chunks, bool add) {
  constexpr unsigned ps = LAYOUT & 2 ? 2048 >> 4 : 32 >> 4, qs = LAYOUT & 1 ? 2048 >> 4 : 32 >> 4;      // 16 of k
  if (chunks >= 4) {
    if constexpr (TERMS == 3) {
#pragma unroll
      for (unsigned c = 0; c < 4; ++c) {
        mma_half<PAIR>(d, pd + c * ps, qd + c * qs + LOW, idesc, c > 0 || add);
        mma_half<PAIR>(d, pd + c * ps + LOW, qd + c * qs, idesc, true);
      }
    }
#pragma unroll
    for (unsigned c = 0; c < 4; ++c) mma_half<PAIR>(d, pd + c * ps, qd + c * qs, idesc, TERMS == 3 || c > 0 || add);
  } else {
    if constexpr (TERMS == 3) {
#pragma unroll 1
      for (unsigned c = 0; c < chunks; ++c) {
        mma_half<PAIR>(d, pd + c * ps, qd + c * qs + LOW, idesc, c > 0 || add);
        mma_half<PAIR>(d, pd + c * ps + LOW, qd + c * qs, idesc, true);
      }
    }
#pragma unroll 1
    for (unsigned c = 0; c < chunks; ++c) mma_half<PAIR>(d, pd + c * ps, qd + c * qs, idesc, TERMS == 3 || c > 0 || add);
  }
}

// The stages of a split of k.
__device__ __forceinline__ void half_range(const HalfPlan& p, unsigned split, unsigned& first, unsigned& last) {
  first = 0;
  last = p.k_stages;
  if (p.splits > 1) {
    first = (unsigned)((uint64_t)p.k_stages * split / p.splits);
    last = (unsigned)((uint64_t)p.k_stages * (split + 1) / p.splits);
  }
}

// SPLIT: few tiles and a long k.  A cluster of CTAs takes one tile, each a part of k; the sums meet in shared memory and are added in
// rank order, each of the eight warps' parts by one of the CTAs.
template <class Epilogue, bool PAIR, int NT, int TERMS, int CHUNK, int LAYOUT, bool SPLIT>
__global__ void __launch_bounds__(kHalfThreads, 1)
half_product_kernel(const __grid_constant__ HalfMaps maps, const HalfPlan p, const __grid_constant__ typename Epilogue::Args args) {
  using S = HalfShape<PAIR, NT, TERMS, CHUNK, Epilogue::kBox>;
  extern __shared__ __align__(1024) unsigned char half_smem[];           // stages, boxes, barriers; the same place in both CTAs
  uint64_t* bars = reinterpret_cast<uint64_t*>(half_smem + S::stages * S::stage_bytes + S::out_bytes);
  unsigned &tmem_base = *reinterpret_cast<unsigned*>(bars + 2 * S::stages + 1 + 16 + 2 * S::accs), &failed = *(&tmem_base + 1);
  const unsigned rank = PAIR ? cluster_rank() : 0;
  const unsigned stage0 = smem_u32(half_smem);
  const unsigned full = smem_u32(bars), empty = full + 8 * S::stages, acc_full = empty + 8 * S::stages, acc_free = acc_full + 8 * S::accs, ended = acc_free + 8 * S::accs, box_full = ended + 8;
  const unsigned warp = threadIdx.x >> 5, lane = threadIdx.x & 31u;
  static_assert(!SPLIT || (!PAIR && NT == 64), "a split tile is one of 128 x 64");
  const unsigned cluster = SPLIT ? p.splits : PAIR ? 2 : 1;
  const unsigned worker = blockIdx.x / cluster, workers = gridDim.x / cluster, part = SPLIT ? cluster_rank() : 0;

  if (threadIdx.x == 0) {
    // while the kernel before this one ends
    prefetch_tensor_map(&maps.p[0]);
    prefetch_tensor_map(&maps.q[0]);
    if (TERMS == 3) prefetch_tensor_map(&maps.p[1]);
    if (TERMS == 3 || p.q_choice) prefetch_tensor_map(&maps.q[1]);
    Epilogue::prefetch(args);
    for (unsigned s = 0; s < S::stages; ++s) {
      mbarrier_init(full + 8 * s, 1);
      mbarrier_init(empty + 8 * s, 1);
    }
    for (unsigned b = 0; b < S::accs; ++b) {
      mbarrier_init(acc_full + 8 * b, 1);
      mbarrier_init(acc_free + 8 * b, PAIR ? 16 : 8);     // one arrival from each of the CTAs' eight epilogue warps
    }
    mbarrier_init(ended, 1);
    for (unsigned b = 0; b < 16; ++b) mbarrier_init(box_full + 8 * b, 1);      // two for each epilogue warp
    mbarrier_init_fence();
    failed = 0;
  }
  // What can be done while the kernel before this one ends: the other CTA's barriers, and the first tile's place (its code is cold).
  HalfPlace start = half_place<PAIR, NT, SPLIT>(worker, p);
  asm volatile("" : "+r"(start.p0), "+r"(start.q0), "+r"(start.matrix), "+r"(start.split), "+r"(start.tile));
  __syncwarp();                                 // the barrier wants whole warps
  if (PAIR) cluster_sync();
  pdl_launch_dependents();
  pdl_wait();                                   // before tensor memory is taken: its last holder has finished
  if (warp == 1) {
    if (PAIR) tmem_alloc_pair(smem_u32(&tmem_base), S::columns);
    else tmem_alloc(smem_u32(&tmem_base), S::columns);
  }
  tcgen05_fence_before();
  __syncthreads();                              // a pair's products begin when both CTAs' operands are there, and so both have come here
  tcgen05_fence_after();
  const unsigned tmem = tmem_base;
  bool ok = true;
  unsigned n = 0;                               // stages so far, over all tiles

  if (warp == 0) {
    if (elect_one()) {
      const CUtensorMap* q_high = p.q_choice && *p.q_choice ? &maps.q[1] : &maps.q[0];
      constexpr bool kPRows = (LAYOUT & 2) != 0, kQRows = (LAYOUT & 1) != 0;
      const unsigned p_loaded = kPRows ? S::p_bytes : p.p_box * 128;
      const unsigned expected = (PAIR ? 2 : 1) * S::parts * (p_loaded + S::q_bytes) + p.starve;
      for (unsigned tile = worker; tile < p.tiles && ok; tile += workers) {
        const HalfPlace at = tile == worker ? start : half_place<PAIR, NT, SPLIT>(tile, p);
        const int p0 = (int)(at.p0 + rank * 128), q0 = (int)(at.q0 + rank * S::q_rows), z = (int)at.matrix;
        unsigned first, last;
        half_range(p, SPLIT ? part : at.split, first, last);
        for (unsigned k = first; k < last; ++k, ++n) {
          const unsigned s = n % S::stages;
          if (n >= S::stages) ok = mbarrier_wait(empty + 8 * s, (n / S::stages - 1) & 1u, kHalfPolls);
          if (!ok) break;
          const unsigned base = stage0 + s * S::stage_bytes;
          const unsigned bar = PAIR ? cluster_address(full + 8 * s, 0) : full + 8 * s;
          if (rank == 0) mbarrier_expect(full + 8 * s, expected);
          const int k0 = (int)(k * 64);
          auto load = [&](unsigned dst, const CUtensorMap* map, int x, int y) {
            if (PAIR) tma_load_3d_pair(dst, map, x, y, z, bar);
            else tma_load_3d(dst, map, x, y, z, bar);
          };
#pragma unroll
          for (unsigned h = 0; h < S::parts; ++h) {
            const unsigned pd = base + h * (S::p_bytes + S::q_bytes), qd = pd + S::p_bytes;
            const CUtensorMap* qm = h == 0 ? q_high : &maps.q[1];
            if (kPRows) {
#pragma unroll
              for (unsigned j = 0; j < 2; ++j) load(pd + j * 8192, &maps.p[h], p0 + (int)(64 * j), k0);
            } else {
              load(pd, &maps.p[h], k0, p0);
            }
            if (kQRows) {
#pragma unroll
              for (unsigned j = 0; j < S::q_rows / 64; ++j) load(qd + j * 8192, qm, q0 + (int)(64 * j), k0);
            } else {
              load(qd, qm, k0, q0);
            }
          }
        }
      }
      // the last stages' commits have to arrive before this CTA may go
      for (unsigned m = n > S::stages ? n - S::stages : 0; m < n && ok; ++m)
        ok = mbarrier_wait(empty + 8 * (m % S::stages), (m / S::stages) & 1u, kHalfPolls);
    }
  } else if (warp == 1) {
    if (rank == 0 && elect_one()) {
      const uint64_t p_desc = half_descriptor(stage0, (LAYOUT & 2) != 0), q_desc = half_descriptor(stage0 + S::p_bytes, (LAYOUT & 1) != 0);
      constexpr unsigned low = (S::p_bytes + S::q_bytes) >> 4;
      unsigned s = 0, parity = 0;
      bool ready = false;                       // the next stage's operands are known to be there
      unsigned t = 0;                           // sums taken so far: of tiles, or of their chunks
      for (unsigned tile = worker; tile < p.tiles && ok; tile += workers) {
        unsigned first, last;
        half_range(p, SPLIT ? part : p.splits > 1 ? tile / p.per_matrix % p.splits : 0, first, last);
        for (unsigned from = first; from < last && ok; ++t) {
          const unsigned to = CHUNK > 0 ? min(last, from + CHUNK) : last;
          const unsigned acc = t % S::accs;
          if (t >= S::accs) ok = PAIR ? mbarrier_wait_cluster(acc_free + 8 * acc, (t / S::accs - 1) & 1u, kHalfPolls)
                                      : mbarrier_wait(acc_free + 8 * acc, (t / S::accs - 1) & 1u, kHalfPolls);
          if (!ok) break;
          tcgen05_fence_after();
          const unsigned d = tmem + acc * NT;
          for (unsigned k = from; k < to; ++k, ++n) {
            ok = ready || mbarrier_wait(full + 8 * s, parity, kHalfPolls);
            if (!ok) break;
            tcgen05_fence_after();
            const unsigned next = s + 1 == S::stages ? 0 : s + 1, next_parity = parity ^ (next == 0);
            ready = mbarrier_test(full + 8 * next, next_parity);    // its answer comes while this stage is issued
            const uint64_t pd = p_desc + s * (S::stage_bytes >> 4), qd = q_desc + s * (S::stage_bytes >> 4);
            half_issue<PAIR, TERMS, LAYOUT, low>(d, pd, qd, p.idesc, p.k_chunks - k * 4, k > from);
            if (PAIR) tcgen05_commit_pair(empty + 8 * s);
            else tcgen05_commit(empty + 8 * s);
            s = next;
            parity = next_parity;
          }
          if (ok) {
            if (PAIR) tcgen05_commit_pair(acc_full + 8 * acc);
            else tcgen05_commit(acc_full + 8 * acc);
          }
          from = to;
        }
      }
      if (!ok) {                                // what was issued has to end before tensor memory is freed; nobody writes it out
        if (PAIR) tcgen05_commit_pair(ended);
        else tcgen05_commit(ended);
        (void)mbarrier_wait(ended, 0, kHalfPolls);
      }
    }
  } else if (warp >= 4) {
    constexpr unsigned kUnits = NT / 64;        // of 32 columns, of this warp
    const unsigned quarter = warp & 3u, odd = warp >= 8;
    const unsigned go = PAIR ? cluster_address(acc_free, 0) : acc_free;
    Epilogue epilogue(args, Box{stage0 + S::stages * S::stage_bytes + (warp - 4) * S::box_bytes, box_full + 16 * (warp - 4), lane});
    unsigned t = 0;
    for (unsigned tile = worker; tile < p.tiles && ok; tile += workers) {
      const HalfPlace at = tile == worker ? start : half_place<PAIR, NT, SPLIT>(tile, p);
      const unsigned row0 = at.p0 + rank * 128 + quarter * 32;
      if (!SPLIT || part == (warp - 4) % cluster) {
        epilogue.begin(args, at, row0, odd);
        if (row0 < p.P && at.q0 + odd * 32 < p.Q) epilogue.ahead(args, at.q0 + odd * 32);
      }
      if constexpr (CHUNK > 0 || SPLIT) {
        constexpr unsigned kTake = CHUNK > 0 ? CHUNK : 1u << 30;
        unsigned first, last;
        half_range(p, SPLIT ? part : at.split, first, last);
        float sum[kUnits][32];
#pragma unroll
        for (unsigned j = 0; j < kUnits; ++j)
#pragma unroll
          for (unsigned q = 0; q < 32; ++q) sum[j][q] = 0.0f;
#pragma unroll 1
        for (unsigned from = first; from < last; from += min(kTake, last - from), ++t) {
          ok = __all_sync(0xFFFFFFFFu, mbarrier_wait(acc_full + 8 * (t % S::accs), (t / S::accs) & 1u, 4 * kHalfPolls + 64 * p.k_stages));
          if (!ok) break;
          tcgen05_fence_after();
          const unsigned lanes = tmem + t % S::accs * NT + (quarter << 21);
          // 16 columns at a time: beside the 128 sums of 256 columns a thread has 40 registers, and epilogues that need more of them keep
          // some of what they hold in local memory (none with StatsEpilogue, 32 to 104 bytes with those of gradients, 92 to 272 with three terms)
#pragma unroll
          for (unsigned j = 0; j < 2 * kUnits; ++j) {
            unsigned v[16];
            tmem_read16(lanes + (odd + j / 2 * 2) * 32 + j % 2 * 16, v);
            if (j + 1 == 2 * kUnits) {
              tcgen05_fence_before();
              __syncwarp();
              if (lane == 0) mbarrier_arrive_cluster(go + 8 * (t % S::accs));
            }
#pragma unroll
            for (unsigned q = 0; q < 16; ++q) sum[j / 2][j % 2 * 16 + q] += __uint_as_float(v[q]);
          }
        }
        if (SPLIT) {
          // all of this CTA's MMAs are done, and with them what its stages held
          if (ok)
#pragma unroll
            for (unsigned q = 0; q < 32; ++q) store_shared4(stage0 + (warp - 4) * 4096 + q * 128 + lane * 4, __float_as_uint(sum[0][q]));
          if (!ok) atomicExch(&failed, 1u);
          break;
        }
        if (!ok) break;
#pragma unroll
        for (unsigned j = 0; j < kUnits; ++j) {
          const unsigned column = at.q0 + (odd + 2 * j) * 32;
          if (j + 1 < kUnits && row0 < p.P && column + 64 < p.Q) epilogue.ahead(args, column + 64);
          if (row0 < p.P && column < p.Q) epilogue.unit(args, column, min(32u, p.Q - column), sum[j]);
          __syncwarp();
        }
      } else {
        ok = __all_sync(0xFFFFFFFFu, mbarrier_wait(acc_full + 8 * (t % S::accs), (t / S::accs) & 1u, 4 * kHalfPolls + 64 * p.k_stages));
        if (!ok) break;
        tcgen05_fence_after();
        const unsigned lanes = tmem + t % S::accs * NT + (quarter << 21);
#pragma unroll 1
        for (unsigned j = 0; j < kUnits; ++j) {
          unsigned v[32];
          tmem_read32(lanes + (odd + 2 * j) * 32, v);
          if (j + 1 == kUnits) {                // this warp's last columns
            tcgen05_fence_before();
            __syncwarp();
            if (lane == 0) mbarrier_arrive_cluster(go + 8 * (t % S::accs));
          }
          float f[32];
#pragma unroll
          for (unsigned q = 0; q < 32; ++q) f[q] = __uint_as_float(v[q]);
          const unsigned column = at.q0 + (odd + 2 * j) * 32;
          if (j + 1 < kUnits && row0 < p.P && column + 64 < p.Q) epilogue.ahead(args, column + 64);
          if (row0 < p.P && column < p.Q) epilogue.unit(args, column, min(32u, p.Q - column), f);
          __syncwarp();
        }
        ++t;
      }
      epilogue.end(args, at, rank * 8 + warp - 4);
      __syncwarp();
      ok = epilogue.box.fine;
    }
    if constexpr (SPLIT) {
      __syncwarp();
      cluster_sync();
      const HalfPlace at = start;
      const unsigned row0 = at.p0 + quarter * 32, column = at.q0 + odd * 32, mine = stage0 + (warp - 4) * 4096 + lane * 4;
      const bool given_up = __any_sync(0xFFFFFFFFu, lane < cluster && load_cluster(cluster_address(smem_u32(&failed), lane)) != 0);
      if (part == (warp - 4) % cluster && !given_up) {
        float sum[32];
#pragma unroll
        for (unsigned q = 0; q < 32; ++q) sum[q] = 0.0f;
        for (unsigned r = 0; r < cluster; ++r) {
          const unsigned from = cluster_address(mine, r);
          float v[32];
#pragma unroll
          for (unsigned q = 0; q < 32; ++q) v[q] = __uint_as_float(load_cluster(from + q * 128));
#pragma unroll
          for (unsigned q = 0; q < 32; ++q) sum[q] = r == 0 ? v[q] : sum[q] + v[q];
        }
        if (row0 < p.P && column < p.Q) epilogue.unit(args, column, min(32u, p.Q - column), sum);
        __syncwarp();
        epilogue.end(args, at, warp - 4);
        __syncwarp();
        ok = ok && epilogue.box.fine;
      }
    }
    epilogue.finish(args);
  }
  if constexpr (SPLIT) {
    if (warp < 4) {
      __syncwarp();
      if (!ok) atomicExch(&failed, 1u);
      __syncwarp();
      cluster_sync();
    }
  }
  if (!ok) atomicExch(&failed, 1u);
  __syncwarp();
  __syncthreads();
  if (failed) {
    // copies that were asked for, here and by the other CTA, have to land before the memory is given up
    if (threadIdx.x == 0) atomicOr(p.status, 1u);
    if (rank == 0 && warp == 0)
      for (unsigned m = n > S::stages ? n - S::stages : 0; m < n; ++m)
        (void)mbarrier_wait(full + 8 * (m % S::stages), (m / S::stages) & 1u, kHalfPolls);
  }
  __syncthreads();
  __syncwarp();
  if (PAIR || SPLIT) cluster_sync();             // nobody leaves while its shared memory is still read
  if (warp == 1) {
    tcgen05_fence_after();
    if (PAIR) tmem_free_pair(tmem, S::columns);
    else tmem_free(tmem, S::columns);
  }
}

// ---------------------------------------------------------------------------------------------------------------------
// Host side.

// Operand `rows` x k of a batch, as its copies see it: stored [rows][ld] (k side by side) or, by_rows, [k][ld].
struct HalfOperand {
  const void* high;
  const void* low;          // TERMS = 3
  size_t ld, batch_stride;  // elements; multiples of eight
  bool by_rows;
};

inline bool half_map(CUtensorMap* map, const void* base, bool bf16, const HalfOperand& o, size_t rows, size_t k, size_t batch, unsigned box_rows) {
  const EncodeTiled f = encode_tiled();
  if (!f) return false;
  const cuuint64_t dims[3] = {o.by_rows ? rows : k, o.by_rows ? k : rows, batch};
  const cuuint64_t strides[2] = {o.ld * 2, (batch > 1 ? o.batch_stride : o.ld) * 2};
  const cuuint32_t box[3] = {64, o.by_rows ? 64u : box_rows, 1}, steps[3] = {1, 1, 1};
  return f(map, bf16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 3, const_cast<void*>(base), dims, strides, box, steps,
           CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

struct HalfProduct {
  HalfOperand p, q;
  const void* q_other;            // another q, rows of stride q_other_ld, taken where *q_choice is not zero
  size_t q_other_ld;
  const unsigned* q_choice;
  size_t P, Q, K, batch;
  bool bf16, symmetric;
  unsigned* status;
  unsigned starve;
};

// A batch of 16-bit matrices as an epilogue's boxes see it: 32 x 32 elements, 64-byte swizzle.
inline bool box_map(CUtensorMap* map, const void* base, bool bf16, size_t rows, size_t cols, size_t ld, size_t batch, size_t batch_stride) {
  const EncodeTiled f = encode_tiled();
  if (!f) return false;
  const cuuint64_t dims[3] = {cols, rows, batch};
  const cuuint64_t strides[2] = {ld * 2, (batch > 1 ? batch_stride : ld) * 2};
  const cuuint32_t box[3] = {32, 32, 1}, steps[3] = {1, 1, 1};
  return f(map, bf16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 3, const_cast<void*>(base), dims, strides, box, steps,
           CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_64B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// Clocks of a product by tiles of a form: rounds of tiles, each its stages, beside a start.  What a stage takes is the tensor cores'
// time (512 clocks for 256 x 256, 64 of k and one term) or shared memory's, 128 bytes a clock, for what the copies write and the
// tensor cores read: 32 + 32, 24 + 24 and 24 + 24 KB for tiles of 256, 128 and 64 columns and one term, 64 + 96, 48 + 72 and 48 + 72 for
// three (measured: 1000 clocks for the last).
struct HalfForm { bool pairs; unsigned nt, split; };      // split: CTAs that share a tile's k, of 128 x 64
inline unsigned long long half_tiles(const HalfProduct& h, unsigned rows, unsigned nt) {
  const unsigned long long tp = (h.P + rows - 1) / rows, tq = (h.Q + nt - 1) / nt;
  if (!h.symmetric) return tp * tq;
  unsigned long long n = 0;
  for (unsigned long long i = 0; i < tp; ++i) n += tq > i * (rows / nt) ? tq - i * (rows / nt) : 0;
  return n;
}
inline HalfForm half_form(const HalfProduct& h, int terms, unsigned splits, int sms, unsigned long long* clocks = nullptr) {
  const unsigned long long stages = (h.K + 63) / 64 / splits + 1, batch = h.batch * splits, pairs = (unsigned)sms / 2;
  const unsigned long long r256 = (half_tiles(h, 256, 256) * batch + pairs - 1) / pairs, r128 = (half_tiles(h, 256, 128) * batch + pairs - 1) / pairs,
                           r64 = (half_tiles(h, 128, 64) * batch + sms - 1) / (unsigned)sms;
  const unsigned s256 = terms == 3 ? 1560 : 530, s128 = terms == 3 ? 980 : 400, s64 = terms == 3 ? 1000 : 390;
  const unsigned long long c256 = r256 * (stages * s256 + 1500) + 6500, c128 = r128 * (stages * s128 + 1200) + 5500, c64 = r64 * (stages * s64 + 1000) + 5000;
  HalfForm best = c256 <= c128 && c256 <= c64 ? HalfForm{true, 256, 1} : c128 <= c64 ? HalfForm{true, 128, 1} : HalfForm{false, 64, 1};
  unsigned long long least = c256 < c128 ? c256 : c128;
  if (c64 < least) least = c64;
  // k shared by a cluster, where all clusters find their place at one time (on 148 SMs two CTAs 72 times, four 32 times, eight 12 times)
  const unsigned long long tiles = half_tiles(h, 128, 64) * batch;
  for (unsigned split = 2; split <= 8 && splits == 1; split *= 2) {
    const unsigned fit = (unsigned)sms * (split == 2 ? 72 : split == 4 ? 32 : 12) / 148;
    if (tiles > fit || stages < 2 * split) break;
    const unsigned long long c = ((h.K + 63) / 64 / split + 1) * s64 + 1000 + 5000 + 2500;
    if (c < least) {
      least = c;
      best = {false, 64, split};
    }
  }
  if (clocks) *clocks = least;
  return best;
}

template <class Epilogue, bool PAIR, int NT, int TERMS, int CHUNK, int LAYOUT, bool SPLIT>
ssgd_status launch_half_form(const HalfProduct& h, const typename Epilogue::Args& args, unsigned splits, int sms, cudaStream_t s) {
  using S = HalfShape<PAIR, NT, TERMS, CHUNK, Epilogue::kBox>;
  HalfPlan p = {};
  const unsigned long long per = half_tiles(h, S::rows, NT), tiles = per * h.batch * (SPLIT ? 1 : splits);
  if (h.P >= (1ull << 31) || h.Q >= (1ull << 31) || h.K >= (1ull << 31) || tiles >= (1ull << 30)) return SSGD_ERR_SIZE;
  p.P = (unsigned)h.P; p.Q = (unsigned)h.Q;
  p.k_stages = (unsigned)((h.K + 63) / 64); p.k_chunks = (unsigned)((h.K + 15) / 16);
  p.tiles_p = (unsigned)((h.P + S::rows - 1) / S::rows); p.tiles_q = (unsigned)((h.Q + NT - 1) / NT);
  p.per_matrix = (unsigned)per; p.tiles = (unsigned)tiles;
  p.splits = splits;
  p.p_box = h.P < 128 ? (unsigned)(h.P + 7) / 8 * 8 : 128;
  p.idesc = mma_half_descriptor(S::rows, NT, h.bf16, h.p.by_rows, h.q.by_rows);
  p.symmetric = h.symmetric;
  p.starve = h.starve;
  p.q_choice = h.q_choice;
  p.status = h.status;
  HalfMaps maps;
  HalfOperand q1 = h.q;
  if (h.q_other) q1.high = h.q_other, q1.ld = h.q_other_ld;
  if (!half_map(&maps.p[0], h.p.high, h.bf16, h.p, h.P, h.K, h.batch, p.p_box) || !half_map(&maps.q[0], h.q.high, h.bf16, h.q, h.Q, h.K, h.batch, S::q_rows))
    return SSGD_ERR_CUDA;
  maps.p[1] = maps.p[0];
  maps.q[1] = maps.q[0];
  if (TERMS == 3 && !half_map(&maps.p[1], h.p.low, h.bf16, h.p, h.P, h.K, h.batch, p.p_box)) return SSGD_ERR_CUDA;
  if ((TERMS == 3 || h.q_other) && !half_map(&maps.q[1], TERMS == 3 ? q1.low : q1.high, h.bf16, q1, h.Q, h.K, h.batch, S::q_rows)) return SSGD_ERR_CUDA;
  auto kernel = half_product_kernel<Epilogue, PAIR, NT, TERMS, CHUNK, LAYOUT, SPLIT>;
  static unsigned long long seen = 0;
  if (!allow_smem(reinterpret_cast<const void*>(kernel), S::smem, &seen)) return SSGD_ERR_CUDA;
  const unsigned long long most = PAIR ? (unsigned)sms / 2 : (unsigned)sms, workers = tiles < most ? tiles : most;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(SPLIT ? splits * tiles : PAIR ? 2 * workers : workers));
  cfg.blockDim = dim3(kHalfThreads);
  cfg.dynamicSmemBytes = S::smem;
  cfg.stream = s;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = SPLIT ? splits : 2;
  attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = PAIR || SPLIT ? 2 : 1;
  (void)cudaLaunchKernelEx(&cfg, kernel, maps, p, args);
  return launch_status();
}

// LAYOUT says what h.p.by_rows and h.q.by_rows say.
template <class Epilogue, int TERMS, int CHUNK, int LAYOUT>
ssgd_status launch_narrow(const HalfProduct& h, const typename Epilogue::Args& args, const HalfForm& form, unsigned splits, int sms, cudaStream_t s) {
  if (form.split > 1) return launch_half_form<Epilogue, false, 64, TERMS, CHUNK, LAYOUT, true>(h, args, form.split, sms, s);
  if (!form.pairs) return launch_half_form<Epilogue, false, 64, TERMS, CHUNK, LAYOUT, false>(h, args, splits, sms, s);
  return launch_half_form<Epilogue, true, 128, TERMS, CHUNK, LAYOUT, false>(h, args, splits, sms, s);
}
template <class Epilogue, int TERMS, int CHUNK, int LAYOUT>
ssgd_status launch_half(const HalfProduct& h, const typename Epilogue::Args& args, const HalfForm& form, unsigned splits, int sms, cudaStream_t s) {
  if (form.nt == 256) return launch_half_form<Epilogue, true, 256, TERMS, CHUNK, LAYOUT, false>(h, args, splits, sms, s);
  return launch_narrow<Epilogue, TERMS, CHUNK, LAYOUT>(h, args, form, splits, sms, s);
}

}  // namespace

#endif  // SSGD_HALF_PRODUCT_CUH_
