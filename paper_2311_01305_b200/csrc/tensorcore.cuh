// Wrappers of the sm_100a instructions behind the tensor-core kernels: tiled bulk copies (TMA) of
// 128-byte-swizzled rows, tcgen05.mma and its completion, TMEM.
#pragma once
#include <cuda.h>

#include "common.cuh"

namespace aweq {

// ------------------------------------------------------------------ host: tensor maps
// A row-major byte matrix [rows x cols], pitch ld bytes (a multiple of 16), read in boxes of box_rows
// rows x 128 bytes, rows swizzled by 128 bytes; what lies outside the matrix reads as zero.
aweq_status tma_bytes_map(CUtensorMap *map, const void *base, long long rows, long long cols, long long ld, int box_rows);

// ------------------------------------------------------------------ device
// Descriptor of an operand tile in shared memory: K-contiguous rows of 128 bytes under the 128-byte swizzle,
// eight rows (1024 bytes) to the next group.  The tile starts on a 1024-byte boundary; 32 bytes
// along K inside the row add 2 to the descriptor.
__device__ __forceinline__ uint64_t tc_desc(uint32_t smem)
{
    return (uint64_t)((smem >> 4) & 0x3fff) | (1ull << 16) | (64ull << 32) | (1ull << 46) | (2ull << 61);
}
// kind::i8, unsigned x unsigned -> int32 (no saturation: sums wrap modulo 2^32), both operands K-major
__host__ __device__ constexpr uint32_t tc_idesc_u8(int m, int n) { return (2u << 4) | ((uint32_t)(n >> 3) << 17) | ((uint32_t)(m >> 4) << 24); }

template <int CG>
__device__ __forceinline__ void tc_alloc(uint32_t *dst, uint32_t cols)
{
    if (CG == 1)
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(dst)), "r"(cols) : "memory");
    else
        asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(dst)), "r"(cols) : "memory");
}
template <int CG>
__device__ __forceinline__ void tc_dealloc(uint32_t tmem, uint32_t cols)
{
    if (CG == 1) {
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(cols) : "memory");
    } else {
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;");
        asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(cols) : "memory");
    }
}
template <int CG>
__device__ __forceinline__ void tc_mma_u8(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, bool add)
{
    if (CG == 1)
        asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %4, 0;\n\t"
                     "tcgen05.mma.cta_group::1.kind::i8 [%0], %1, %2, %3, p;\n\t}"
                     ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"((uint32_t)add) : "memory");
    else
        asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %4, 0;\n\t"
                     "tcgen05.mma.cta_group::2.kind::i8 [%0], %1, %2, %3, p;\n\t}"
                     ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"((uint32_t)add) : "memory");
}
// one arrival on the barrier (cta_group::2: on that barrier of both CTAs of the pair) when every
// tcgen05.mma issued so far by this thread has completed
template <int CG>
__device__ __forceinline__ void tc_commit(uint64_t *bar)
{
    if (CG == 1)
        asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(smem_u32(bar)) : "memory");
    else
        asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;"
                     ::"r"(smem_u32(bar)), "h"((uint16_t)3) : "memory");
}
__device__ __forceinline__ void tc_fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tc_fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tc_wait_ld() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }

// 32 lanes x 32 columns of TMEM: lane l of the warp gets the 32 values of TMEM lane (its quarter) + l
__device__ __forceinline__ void tc_ld32(uint32_t tmem, uint32_t (&r)[32])
{
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 "
        "{%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]),
          "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]), "=r"(r[17]), "=r"(r[18]),
          "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]),
          "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
        : "r"(tmem));
}

// 2-D box global -> this CTA's shared memory.  CG 2: the barrier may be the pair's other CTA's
// (bar is a shared::cluster address either way).
template <int CG>
__device__ __forceinline__ void tma_load2(uint32_t dst, const CUtensorMap *map, int x, int y, uint32_t bar)
{
    if (CG == 1)
        asm volatile("cp.async.bulk.tensor.2d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];"
                     ::"r"(dst), "l"(map), "r"(x), "r"(y), "r"(bar) : "memory");
    else
        asm volatile("cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];"
                     ::"r"(dst), "l"(map), "r"(x), "r"(y), "r"(bar) : "memory");
}
__device__ __forceinline__ void tma_prefetch_map(const CUtensorMap *map)
{
    asm volatile("prefetch.tensormap [%0];" ::"l"(map) : "memory");
}

}  // namespace aweq
