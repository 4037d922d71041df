// The sm_100a instructions that the 4-bit product is written in: mbarriers, bulk and tiled asynchronous copies, tensor
// memory, block-scaled tcgen05.mma.  One wrapper per instruction, no policy except that every wait is bounded.
#ifndef SSGD_SM100_CUH_
#define SSGD_SM100_CUH_

#include <cuda.h>
#include <cuda_runtime.h>
#include <stdint.h>

namespace {

__device__ __forceinline__ unsigned smem_u32(const void* p) { return (unsigned)__cvta_generic_to_shared(p); }

__device__ __forceinline__ void mbarrier_init(unsigned bar, unsigned count) {
  asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(count) : "memory");
}
__device__ __forceinline__ void mbarrier_init_fence() { asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory"); }
__device__ __forceinline__ void mbarrier_expect(unsigned bar, unsigned bytes) {
  asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
}
__device__ __forceinline__ void mbarrier_arrive(unsigned bar) {
  asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory");
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
// 16 columns of this warp's 32 lanes, one lane per thread.
__device__ __forceinline__ void tmem_load16(unsigned tmem, unsigned (&v)[16]) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
      : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7]), "=r"(v[8]), "=r"(v[9]),
        "=r"(v[10]), "=r"(v[11]), "=r"(v[12]), "=r"(v[13]), "=r"(v[14]), "=r"(v[15])
      : "r"(tmem));
}
// Loads are complete after this; the values pass through it so that no use of them can be moved ahead of it.
__device__ __forceinline__ void tmem_load_wait(unsigned (&v)[16]) {
  asm volatile("tcgen05.wait::ld.sync.aligned;"
               : "+r"(v[0]), "+r"(v[1]), "+r"(v[2]), "+r"(v[3]), "+r"(v[4]), "+r"(v[5]), "+r"(v[6]), "+r"(v[7]), "+r"(v[8]), "+r"(v[9]),
                 "+r"(v[10]), "+r"(v[11]), "+r"(v[12]), "+r"(v[13]), "+r"(v[14]), "+r"(v[15])::"memory");
}

// 512 bytes, a tile of block scales, to four columns, the same in each 32 lanes.
__device__ __forceinline__ void tcgen05_copy_scales(unsigned tmem, uint64_t desc) {
  asm volatile("tcgen05.cp.cta_group::1.32x128b.warpx4 [%0], %1;" ::"r"(tmem), "l"(desc) : "memory");
}

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

}  // namespace

#endif  // SSGD_SM100_CUH_
