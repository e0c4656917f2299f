// tcgen05 wrappers (5th-generation tensor cores, tensor memory).
#pragma once
#include "gms_ptx.h"

namespace gms {
namespace ptx {

// Shared-memory operand descriptor, 128-byte swizzle, as two words; (offset >> 4) may be added to the low one.
// K-major operands: `sbo` bytes between groups of 8 rows (lbo unused).
// MN-major operands: `lbo` bytes between groups of 64 elements, `sbo` bytes between groups of 8 k.
__host__ __device__ constexpr uint32_t desc_lo(uint32_t addr, uint32_t lbo) { return (addr >> 4 & 0x3fffu) | (lbo >> 4 & 0x3fffu) << 16; }
__host__ __device__ constexpr uint32_t desc_hi(uint32_t sbo) { return (sbo >> 4 & 0x3fffu) | 1u << 14 | 2u << 29; }
// kind::f16 instruction descriptor: 32-bit accumulators, A K-major; `bf16` else f16, `b_mn` B is MN-major.
__host__ __device__ constexpr uint32_t f16_idesc(uint32_t m, uint32_t n, bool bf16, bool b_mn)
{
    return 1u << 4 | (bf16 ? 1u : 0u) << 7 | (bf16 ? 1u : 0u) << 10 | (b_mn ? 1u : 0u) << 16 | (n >> 3) << 17 | (m >> 4) << 24;
}
// The instructions below are issued by one lane of a warp whose lanes all get here with the same operands: `on` is 1 in that
// lane (see one_lane).  Kept out of a branch on the lane, the operands stay in uniform registers.
__device__ __forceinline__ uint32_t one_lane()
{
    uint32_t on;
    asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(on));
    return on;
}
// d (tensor memory) = a b (+ d), a in shared memory.  Descriptors as low words; the high word is shared.
__device__ __forceinline__ void mma_ss(uint32_t on, uint32_t d, uint32_t a, uint32_t b, uint32_t hi, uint32_t idesc, bool add)
{
    asm volatile(
        "{\n\t.reg .pred p, q;\n\t.reg .b64 da, db;\n\tsetp.ne.u32 q, %0, 0;\n\tsetp.ne.u32 p, %6, 0;\n\t"
        "mov.b64 da, {%2, %4};\n\tmov.b64 db, {%3, %4};\n\t"
        "@q tcgen05.mma.cta_group::1.kind::f16 [%1], da, db, %5, p;\n\t}" ::"r"(on),
        "r"(d), "r"(a), "r"(b), "r"(hi), "r"(idesc), "r"((uint32_t)add)
        : "memory");
}
// The same with a in tensor memory (two 16-bit elements a column).
__device__ __forceinline__ void mma_ts(uint32_t on, uint32_t d, uint32_t a, uint32_t b, uint32_t hi, uint32_t idesc, bool add)
{
    asm volatile(
        "{\n\t.reg .pred p, q;\n\t.reg .b64 db;\n\tsetp.ne.u32 q, %0, 0;\n\tsetp.ne.u32 p, %6, 0;\n\t"
        "mov.b64 db, {%3, %4};\n\t"
        "@q tcgen05.mma.cta_group::1.kind::f16 [%1], [%2], db, %5, p;\n\t}" ::"r"(on),
        "r"(d), "r"(a), "r"(b), "r"(hi), "r"(idesc), "r"((uint32_t)add)
        : "memory");
}
// One arrival on `bar` once everything this lane has issued to the tensor core is done.
__device__ __forceinline__ void tc_commit(uint32_t on, uint32_t bar)
{
    asm volatile(
        "{\n\t.reg .pred q;\n\tsetp.ne.u32 q, %0, 0;\n\t"
        "@q tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%1];\n\t}" ::"r"(on),
        "r"(bar)
        : "memory");
}
__device__ __forceinline__ void tc_fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tc_fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tmem_alloc(uint32_t smem_slot, uint32_t cols)
{
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_slot), "r"(cols) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
}
__device__ __forceinline__ void tmem_free(uint32_t addr, uint32_t cols)
{
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(addr), "r"(cols) : "memory");
}
__device__ __forceinline__ void tmem_wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

// 32 columns of the warp's 32 lanes (lane = row).  tmem_ld32 starts the load; the registers may be used after
// tmem_wait32 has been given them.
__device__ __forceinline__ void tmem_ld32(uint32_t addr, uint32_t *r)
{
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
                 "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]),
                   "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]),
                   "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]),
                   "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
                 : "r"(addr));
}
__device__ __forceinline__ void tmem_wait32(uint32_t *r)
{
    asm volatile("tcgen05.wait::ld.sync.aligned;"
                 : "+r"(r[0]), "+r"(r[1]), "+r"(r[2]), "+r"(r[3]), "+r"(r[4]), "+r"(r[5]), "+r"(r[6]), "+r"(r[7]), "+r"(r[8]),
                   "+r"(r[9]), "+r"(r[10]), "+r"(r[11]), "+r"(r[12]), "+r"(r[13]), "+r"(r[14]), "+r"(r[15]), "+r"(r[16]),
                   "+r"(r[17]), "+r"(r[18]), "+r"(r[19]), "+r"(r[20]), "+r"(r[21]), "+r"(r[22]), "+r"(r[23]), "+r"(r[24]),
                   "+r"(r[25]), "+r"(r[26]), "+r"(r[27]), "+r"(r[28]), "+r"(r[29]), "+r"(r[30]), "+r"(r[31])
                 :
                 : "memory");
}
__device__ __forceinline__ void tmem_st32(uint32_t addr, const uint32_t *r)
{
    asm volatile("tcgen05.st.sync.aligned.32x32b.x32.b32 [%32], {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
                 "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31};" ::"r"(r[0]),
                   "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]),
                   "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(r[16]), "r"(r[17]), "r"(r[18]),
                   "r"(r[19]), "r"(r[20]), "r"(r[21]), "r"(r[22]), "r"(r[23]), "r"(r[24]), "r"(r[25]), "r"(r[26]), "r"(r[27]),
                   "r"(r[28]), "r"(r[29]), "r"(r[30]), "r"(r[31]), "r"(addr)
                 : "memory");
}

}  // namespace ptx
}  // namespace gms
