// The sm_100a instructions that the products are written in: mbarriers, bulk and tiled asynchronous copies, tensor
// memory, tcgen05.mma of 16-bit and of block-scaled 4-bit operands.  One wrapper per instruction, no policy except that every wait is bounded.
#ifndef SSGD_SM100_CUH_
#define SSGD_SM100_CUH_

#include <cuda.h>
#include <cuda_runtime.h>
#include <stdint.h>

namespace {

__device__ __forceinline__ unsigned smem_u32(const void* p) { return (unsigned)__cvta_generic_to_shared(p); }

// True in one thread of a whole warp, always the same one.  What a branch on it holds is known to run once, so that operands
// of the tensor-core instructions go to uniform registers directly; behind `lane == 0` each of them costs 66-78 clocks to
// issue (B200: four MMAs of 256 x 256 x 64 with twelve scale copies 1143 clocks, elected 516).
__device__ __forceinline__ bool elect_one() {
  unsigned e;
  asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(e));
  return e != 0;
}

__device__ __forceinline__ void mbarrier_init(unsigned bar, unsigned count) {
  asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(count) : "memory");
}
__device__ __forceinline__ void mbarrier_init_fence() { asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory"); }
__device__ __forceinline__ void mbarrier_expect(unsigned bar, unsigned bytes) {
  asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
}
// One poll, suspended by the hardware for about a microsecond at most.
__device__ __forceinline__ bool mbarrier_poll(unsigned bar, unsigned parity) {
  unsigned done;
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2, %3;\n\t"
      "selp.u32 %0, 1, 0, p;\n\t}"
      : "=r"(done)
      : "r"(bar), "r"(parity), "r"(1000u)
      : "memory");
  return done != 0;
}
// The same without suspension: what is true now.
__device__ __forceinline__ bool mbarrier_test(unsigned bar, unsigned parity) {
  unsigned done;
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "mbarrier.test_wait.parity.shared::cta.b64 p, [%1], %2;\n\t"
      "selp.u32 %0, 1, 0, p;\n\t}"
      : "=r"(done)
      : "r"(bar), "r"(parity)
      : "memory");
  return done != 0;
}
// Waits for the phase of the given parity; false when it has not completed within `polls` polls.
__device__ __forceinline__ bool mbarrier_wait(unsigned bar, unsigned parity, unsigned polls) {
  for (unsigned i = 0; i < polls; ++i)
    if (mbarrier_poll(bar, parity)) return true;
  return false;
}

// Box of a two-dimensional tensor to shared memory; x is a multiple of 16 bytes.
__device__ __forceinline__ void tma_load_2d(unsigned dst, const CUtensorMap* map, int x, int y, unsigned bar) {
  asm volatile("cp.async.bulk.tensor.2d.shared::cta.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];"
               ::"r"(dst), "l"(map), "r"(x), "r"(y), "r"(bar)
               : "memory");
}
// A box from shared memory to a two-dimensional tensor, what lies outside it left out; x is a multiple of 16 bytes.  The
// copies of a thread form groups: it can wait until the last group has read its shared memory, or is complete.
__device__ __forceinline__ void tma_store_2d(const CUtensorMap* map, int x, int y, unsigned src) {
  asm volatile("cp.async.bulk.tensor.2d.global.shared::cta.tile.bulk_group [%0, {%1, %2}], [%3];\n\tcp.async.bulk.commit_group;"
               ::"l"(map), "r"(x), "r"(y), "r"(src)
               : "memory");
}
__device__ __forceinline__ void tma_store_3d(const CUtensorMap* map, int x, int y, int z, unsigned src) {
  asm volatile("cp.async.bulk.tensor.3d.global.shared::cta.tile.bulk_group [%0, {%1, %2, %3}], [%4];\n\tcp.async.bulk.commit_group;"
               ::"l"(map), "r"(x), "r"(y), "r"(z), "r"(src)
               : "memory");
}
// All groups but the last one.
__device__ __forceinline__ void tma_store_wait_read_but_last() { asm volatile("cp.async.bulk.wait_group.read 1;" ::: "memory"); }
__device__ __forceinline__ void tma_store_wait_read() { asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory"); }
__device__ __forceinline__ void tma_store_wait() { asm volatile("cp.async.bulk.wait_group 0;" ::: "memory"); }
// Ordinary writes to shared memory before this are seen by asynchronous copies after it.
__device__ __forceinline__ void async_proxy_fence() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }
// The same for all memory: asynchronous copies on one side of a barrier, and asynchronous copies on the other.
__device__ __forceinline__ void proxy_fence() { asm volatile("fence.proxy.async;" ::: "memory"); }
__device__ __forceinline__ void store_shared16(unsigned at, unsigned a, unsigned b, unsigned c, unsigned d) {
  asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(at), "r"(a), "r"(b), "r"(c), "r"(d) : "memory");
}
// `bytes` (a multiple of 16) from a 16-byte aligned address to shared memory.
__device__ __forceinline__ void bulk_copy(unsigned dst, const void* src, unsigned bytes, unsigned bar) {
  asm volatile("cp.async.bulk.shared::cta.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];"
               ::"r"(dst), "l"(src), "r"(bytes), "r"(bar)
               : "memory");
}
__device__ __forceinline__ void prefetch_tensor_map(const CUtensorMap* map) {
  asm volatile("prefetch.tensormap [%0];" ::"l"(map) : "memory");
}

// Tensor memory: 128 lanes x 512 columns of 32 bits; an address is lane << 16 | column.  A whole warp allocates a power of
// two of columns (32 or more) and frees them again.
__device__ __forceinline__ void tmem_alloc(unsigned where, unsigned columns) {
  asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(where), "r"(columns) : "memory");
  asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
}
__device__ __forceinline__ void tmem_free(unsigned tmem, unsigned columns) {
  asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(columns) : "memory");
}
__device__ __forceinline__ void tcgen05_fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tcgen05_fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
// The mbarrier gets one arrival when all tcgen05 work that this thread has issued is done.
__device__ __forceinline__ void tcgen05_commit(unsigned bar) {
  asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
}
// 32 columns of this warp's 32 lanes, complete on return.
__device__ __forceinline__ void tmem_read32(unsigned tmem, unsigned (&v)[32]) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
      "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];\n\t"
      "tcgen05.wait::ld.sync.aligned;"
      : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7]), "=r"(v[8]), "=r"(v[9]),
        "=r"(v[10]), "=r"(v[11]), "=r"(v[12]), "=r"(v[13]), "=r"(v[14]), "=r"(v[15]), "=r"(v[16]), "=r"(v[17]), "=r"(v[18]), "=r"(v[19]),
        "=r"(v[20]), "=r"(v[21]), "=r"(v[22]), "=r"(v[23]), "=r"(v[24]), "=r"(v[25]), "=r"(v[26]), "=r"(v[27]), "=r"(v[28]), "=r"(v[29]),
        "=r"(v[30]), "=r"(v[31])
      : "r"(tmem)
      : "memory");
}

__device__ __forceinline__ void tmem_read16(unsigned tmem, unsigned (&v)[16]) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];\n\t"
      "tcgen05.wait::ld.sync.aligned;"
      : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7]), "=r"(v[8]), "=r"(v[9]),
        "=r"(v[10]), "=r"(v[11]), "=r"(v[12]), "=r"(v[13]), "=r"(v[14]), "=r"(v[15])
      : "r"(tmem)
      : "memory");
}

// 512 bytes, a tile of block scales, to four columns, the same in each 32 lanes.
__device__ __forceinline__ void tcgen05_copy_scales(unsigned tmem, uint64_t desc) {
  asm volatile("tcgen05.cp.cta_group::1.32x128b.warpx4 [%0], %1;" ::"r"(tmem), "l"(desc) : "memory");
}

__device__ __forceinline__ void store_shared4(unsigned at, unsigned v) { asm volatile("st.shared.b32 [%0], %1;" ::"r"(at), "r"(v) : "memory"); }

// Shared-memory matrix descriptor: start address, stride between groups of eight rows, layout (0: none, 2: 128-byte swizzle).
__device__ __forceinline__ uint64_t smem_descriptor(unsigned addr, unsigned group_stride, unsigned layout) {
  return (uint64_t)((addr & 0x3FFFFu) >> 4) | (uint64_t)1 << 16 | (uint64_t)(group_stride >> 4) << 32 | (uint64_t)1 << 46 | (uint64_t)layout << 61;
}

// D[128 x n] (+)= A[128 x 64] B[n x 64]^T of 4-bit operands with block scales in tensor memory.  E8M0 scales of 32 values
// (kind::mxf4) or E4M3 scales of 16 (kind::mxf4nvf4).
template <bool E8M0>
__device__ __forceinline__ void mma_fp4(unsigned d, uint64_t a, uint64_t b, unsigned idesc, unsigned a_scales, unsigned b_scales, bool add) {
  if constexpr (E8M0)
    asm volatile(
        "{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %6, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::mxf4.block_scale.scale_vec::2X [%0], %1, %2, %3, [%4], [%5], p;\n\t}"
        ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(a_scales), "r"(b_scales), "r"((unsigned)add)
        : "memory");
  else
    asm volatile(
        "{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %6, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::mxf4nvf4.block_scale.scale_vec::4X [%0], %1, %2, %3, [%4], [%5], p;\n\t}"
        ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(a_scales), "r"(b_scales), "r"((unsigned)add)
        : "memory");
}
// Instruction descriptor: E2M1 operands, both k-major; n columns, m rows; scale type; which half of a scale word (0 or 2).
__device__ __forceinline__ unsigned mma_fp4_descriptor(unsigned m, unsigned n, bool e8m0, unsigned scale_id) {
  return scale_id << 4 | 1u << 7 | 1u << 10 | (n >> 3) << 17 | (e8m0 ? 1u << 23 : 0u) | (m >> 4) << 24 | scale_id << 29;
}

// D[m x n] (+)= A[m x 16] B[n x 16]^T of 16-bit operands, by one CTA (m = 128) or a pair (m = 256, see below).
template <bool PAIR>
__device__ __forceinline__ void mma_half(unsigned d, uint64_t a, uint64_t b, unsigned idesc, bool add) {
  if constexpr (PAIR)
    asm volatile(
        "{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n\t}"
        ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"((unsigned)add)
        : "memory");
  else
    asm volatile(
        "{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}"
        ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"((unsigned)add)
        : "memory");
}
// Instruction descriptor: fp32 accumulators; both operands bf16 or both fp16; whether each lies with its rows (m, n) side by side
// instead of its k.
__host__ __device__ constexpr unsigned mma_half_descriptor(unsigned m, unsigned n, bool bf16, bool a_by_rows, bool b_by_rows) {
  return 1u << 4 | (bf16 ? 1u << 7 | 1u << 10 : 0u) | (a_by_rows ? 1u << 15 : 0u) | (b_by_rows ? 1u << 16 : 0u) | (n >> 3) << 17 | (m >> 4) << 24;
}
// Descriptor of a 16-bit operand in shared memory as tiled copies of 128-byte rows leave it (128-byte swizzle).  A row holds 64
// of k (groups of eight rows 1024 bytes apart); or, the operand lying by rows, 64 of its rows for one k: eight k 1024 bytes
// apart, the next 64 rows `next_rows` bytes.
__device__ __forceinline__ uint64_t half_descriptor(unsigned addr, bool by_rows, unsigned next_rows = 8192) {
  return (uint64_t)((addr & 0x3FFFFu) >> 4) | (uint64_t)(by_rows ? next_rows >> 4 : 1) << 16 | (uint64_t)(1024 >> 4) << 32 | (uint64_t)1 << 46 | (uint64_t)2 << 61;
}
// Box of a three-dimensional tensor to shared memory; x is a multiple of 16 bytes.
__device__ __forceinline__ void tma_load_3d(unsigned dst, const CUtensorMap* map, int x, int y, int z, unsigned bar) {
  asm volatile("cp.async.bulk.tensor.3d.shared::cta.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];"
               ::"r"(dst), "l"(map), "r"(x), "r"(y), "r"(z), "r"(bar)
               : "memory");
}

// ---------------------------------------------------------------------------------------------------------------------
// Two CTAs of a cluster as one unit (cta_group::2): one thread of the first CTA issues for both; an MMA has 256 rows, 128
// from each CTA, and takes half of its n rows from each; each CTA holds its half of D, and the scales it needs.

__device__ __forceinline__ unsigned cluster_rank() {
  unsigned r;
  asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
  return r;
}
__device__ __forceinline__ unsigned cluster_size() {
  unsigned r;
  asm volatile("mov.u32 %0, %%cluster_nctarank;" : "=r"(r));
  return r;
}
__device__ __forceinline__ unsigned cluster_address(unsigned addr, unsigned rank) {   // of the same place in another CTA
  unsigned out;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(out) : "r"(addr), "r"(rank));
  return out;
}
__device__ __forceinline__ void cluster_sync() {
  asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
__device__ __forceinline__ unsigned load_cluster(unsigned cluster_addr) {          // from another CTA's shared memory
  unsigned v;
  asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(v) : "r"(cluster_addr) : "memory");
  return v;
}
// An arrival at a barrier of another CTA that orders tensor memory only (between the two tcgen05 fences): relaxed, since a
// release would first wait for all of this thread's stores to global memory (a third of the time of a short product).
__device__ __forceinline__ void mbarrier_arrive_cluster(unsigned cluster_bar) {
  asm volatile("mbarrier.arrive.relaxed.cluster.shared::cluster.b64 _, [%0];" ::"r"(cluster_bar) : "memory");
}
// Like mbarrier_wait, for such arrivals.
__device__ __forceinline__ bool mbarrier_wait_cluster(unsigned bar, unsigned parity, unsigned polls) {
  for (unsigned i = 0; i < polls; ++i) {
    unsigned done;
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "mbarrier.try_wait.parity.relaxed.cluster.shared::cta.b64 p, [%1], %2, %3;\n\t"
        "selp.u32 %0, 1, 0, p;\n\t}"
        : "=r"(done)
        : "r"(bar), "r"(parity), "r"(1000u)
        : "memory");
    if (done) return true;
  }
  return false;
}
// The box goes to this CTA's memory, its bytes are counted on a barrier of either CTA.
__device__ __forceinline__ void tma_load_2d_pair(unsigned dst, const CUtensorMap* map, int x, int y, unsigned cluster_bar) {
  asm volatile("cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];"
               ::"r"(dst), "l"(map), "r"(x), "r"(y), "r"(cluster_bar)
               : "memory");
}
__device__ __forceinline__ void tma_load_3d_pair(unsigned dst, const CUtensorMap* map, int x, int y, int z, unsigned cluster_bar) {
  asm volatile("cp.async.bulk.tensor.3d.cta_group::2.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];"
               ::"r"(dst), "l"(map), "r"(x), "r"(y), "r"(z), "r"(cluster_bar)
               : "memory");
}
__device__ __forceinline__ void tmem_alloc_pair(unsigned where, unsigned columns) {
  asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(where), "r"(columns) : "memory");
  asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
}
__device__ __forceinline__ void tmem_free_pair(unsigned tmem, unsigned columns) {
  asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(columns) : "memory");
}
// One arrival at the same barrier of both CTAs when all tcgen05 work of this thread is done.
__device__ __forceinline__ void tcgen05_commit_pair(unsigned bar) {
  asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;"
               ::"r"(bar), "h"((uint16_t)3)
               : "memory");
}
__device__ __forceinline__ void tcgen05_copy_scales_pair(unsigned tmem, uint64_t desc) {
  asm volatile("tcgen05.cp.cta_group::2.32x128b.warpx4 [%0], %1;" ::"r"(tmem), "l"(desc) : "memory");
}
template <bool E8M0>
__device__ __forceinline__ void mma_fp4_pair(unsigned d, uint64_t a, uint64_t b, unsigned idesc, unsigned a_scales, unsigned b_scales, bool add) {
  if constexpr (E8M0)
    asm volatile(
        "{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %6, 0;\n\t"
        "tcgen05.mma.cta_group::2.kind::mxf4.block_scale.scale_vec::2X [%0], %1, %2, %3, [%4], [%5], p;\n\t}"
        ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(a_scales), "r"(b_scales), "r"((unsigned)add)
        : "memory");
  else
    asm volatile(
        "{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %6, 0;\n\t"
        "tcgen05.mma.cta_group::2.kind::mxf4nvf4.block_scale.scale_vec::4X [%0], %1, %2, %3, [%4], [%5], p;\n\t}"
        ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(a_scales), "r"(b_scales), "r"((unsigned)add)
        : "memory");
}
}  // namespace

#endif  // SSGD_SM100_CUH_
