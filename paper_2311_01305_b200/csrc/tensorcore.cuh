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
// A pool of 16-bit pages [pages x tokens x heads x dim] with any strides (elements, multiples of 8), read in boxes of
// box_tokens tokens x 64 elements of one head, rows swizzled by 128 bytes; elements past head_dim read as zero.
// Strides of 2^40 bytes and more do not fit a tensor map.
inline bool tma_pool_fits(long long page_stride, long long token_stride, long long head_stride)
{
    return page_stride < 1ll << 39 && token_stride < 1ll << 39 && head_stride < 1ll << 39;
}
// `tiles` tiles of 512 bytes in a row, read `box` at a time into consecutive shared memory
aweq_status tma_tiles_map(CUtensorMap *map, const void *base, long long tiles, int box);
// 16-bit rows [tokens x heads x dim], pitch ld elements (heads side by side), read in boxes of box_tokens tokens x box_heads heads x
// 64 elements, swizzled by 128 bytes; elements past dim and tokens past the last read as zero
aweq_status tma_heads_map(CUtensorMap *map, const void *base, long long tokens, int heads, int dim, long long ld, int box_heads, int box_tokens);
aweq_status tma_pool_map(CUtensorMap *map, const void *base, long long pages, int tokens, int heads, int dim, long long page_stride,
                         long long token_stride, long long head_stride, int box_tokens);

// ------------------------------------------------------------------ device
// Descriptor of an operand tile in shared memory, as two words: K-contiguous rows of 128 bytes under the 128-byte swizzle,
// eight rows (1024 bytes) to the next group.  The tile starts on a 1024-byte boundary; 32 bytes along K inside the
// row add 2 to the low word, other offsets of the tile their 16-byte units.
constexpr uint32_t kTcDescHi = 64u | (1u << 14) | (2u << 29);
__device__ __forceinline__ uint32_t tc_desc(uint32_t smem) { return ((smem >> 4) & 0x3fff) | (1u << 16); }
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
// The warp that issues products runs as one: every lane computes the same operands (so that they live in uniform registers;
// with a single lane in a branch of its own each instruction took about 130 cycles to issue), and `lead` picks the lane
// that the instruction is for.
__device__ __forceinline__ bool tc_elect()
{
    uint32_t ok;
    asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(ok));
    return ok != 0;
}
template <int CG>
__device__ __forceinline__ void tc_mma_u8(uint32_t d, uint32_t a, uint32_t b, uint32_t idesc, bool add, bool lead)
{
    if (CG == 1)
        asm volatile("{\n\t.reg .pred p, q;\n\t.reg .b64 da, db;\n\tsetp.ne.u32 p, %4, 0;\n\tsetp.ne.u32 q, %6, 0;\n\t"
                     "mov.b64 da, {%1, %5};\n\tmov.b64 db, {%2, %5};\n\t"
                     "@q tcgen05.mma.cta_group::1.kind::i8 [%0], da, db, %3, p;\n\t}"
                     ::"r"(d), "r"(a), "r"(b), "r"(idesc), "r"((uint32_t)add), "r"(kTcDescHi), "r"((uint32_t)lead) : "memory");
    else
        asm volatile("{\n\t.reg .pred p, q;\n\t.reg .b64 da, db;\n\tsetp.ne.u32 p, %4, 0;\n\tsetp.ne.u32 q, %6, 0;\n\t"
                     "mov.b64 da, {%1, %5};\n\tmov.b64 db, {%2, %5};\n\t"
                     "@q tcgen05.mma.cta_group::2.kind::i8 [%0], da, db, %3, p;\n\t}"
                     ::"r"(d), "r"(a), "r"(b), "r"(idesc), "r"((uint32_t)add), "r"(kTcDescHi), "r"((uint32_t)lead) : "memory");
}
// ------------------------------------------------------------------ 4-bit operands with block scales
// e2m1 x e2m1 -> binary32, both K-major, 64 elements of K (32 bytes of a row) an instruction.  `e8m0`: blocks of 32 with
// power-of-two scales, of which a word of TMEM holds those of two instructions; else blocks of 16 with e4m3 scales, a word
// for one.  `half`: which two of the four scales (e8m0).
__host__ __device__ constexpr uint32_t tc_idesc_mx4(bool e8m0, int m, int n)
{
    return (1u << 7) | (1u << 10) | ((uint32_t)(n >> 3) << 17) | ((e8m0 ? 1u : 0u) << 23) | ((uint32_t)(m >> 4) << 24);
}
__device__ __forceinline__ uint32_t tc_idesc_mx4_half(uint32_t idesc, int half) { return idesc | ((uint32_t)half << 5) | ((uint32_t)half << 30); }
template <int CG, bool E8M0>
__device__ __forceinline__ void tc_mma_mx4(uint32_t d, uint32_t a, uint32_t b, uint32_t idesc, uint32_t sa, uint32_t sb, bool add, bool lead)
{
#define AWEQ_MMA_MX4(CG_, KIND_)                                                                                              \
    asm volatile("{\n\t.reg .pred p, q;\n\t.reg .b64 da, db;\n\tsetp.ne.u32 p, %4, 0;\n\tsetp.ne.u32 q, %6, 0;\n\t"           \
                 "mov.b64 da, {%1, %5};\n\tmov.b64 db, {%2, %5};\n\t"                                                        \
                 "@q tcgen05.mma.cta_group::" CG_ "." KIND_ " [%0], da, db, %3, [%7], [%8], p;\n\t}"                          \
                 ::"r"(d), "r"(a), "r"(b), "r"(idesc), "r"((uint32_t)add), "r"(kTcDescHi), "r"((uint32_t)lead), "r"(sa), "r"(sb) : "memory")
    if (CG == 1) {
        if (E8M0) AWEQ_MMA_MX4("1", "kind::mxf4.block_scale.scale_vec::2X");
        else AWEQ_MMA_MX4("1", "kind::mxf4nvf4.block_scale.scale_vec::4X");
    } else {
        if (E8M0) AWEQ_MMA_MX4("2", "kind::mxf4.block_scale.scale_vec::2X");
        else AWEQ_MMA_MX4("2", "kind::mxf4nvf4.block_scale.scale_vec::4X");
    }
#undef AWEQ_MMA_MX4
}
// A tile of scales (32 rows of 16 bytes, without swizzle) to four columns of TMEM, the same in every quarter of the lanes.  In order
// with the products that this thread issues later; not with those before it.
constexpr uint32_t kTcScaleDescHi = 8u | (1u << 14);
template <int CG>
__device__ __forceinline__ void tc_copy_scales(uint32_t tmem, uint32_t smem, bool lead)
{
    const uint32_t lo = (smem >> 4) & 0x3fff;
    if (CG == 1)
        asm volatile("{\n\t.reg .pred q;\n\t.reg .b64 d;\n\tsetp.ne.u32 q, %3, 0;\n\tmov.b64 d, {%1, %2};\n\t"
                     "@q tcgen05.cp.cta_group::1.32x128b.warpx4 [%0], d;\n\t}" ::"r"(tmem), "r"(lo), "r"(kTcScaleDescHi), "r"((uint32_t)lead) : "memory");
    else
        asm volatile("{\n\t.reg .pred q;\n\t.reg .b64 d;\n\tsetp.ne.u32 q, %3, 0;\n\tmov.b64 d, {%1, %2};\n\t"
                     "@q tcgen05.cp.cta_group::2.32x128b.warpx4 [%0], d;\n\t}" ::"r"(tmem), "r"(lo), "r"(kTcScaleDescHi), "r"((uint32_t)lead) : "memory");
}
// one arrival on the barrier (cta_group::2: on that barrier of both CTAs of the pair) when every
// tcgen05.mma issued so far by this thread has completed
template <int CG>
__device__ __forceinline__ void tc_commit(uint64_t *bar, bool lead)
{
    if (CG == 1)
        asm volatile("{\n\t.reg .pred q;\n\tsetp.ne.u32 q, %1, 0;\n\t"
                     "@q tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];\n\t}"
                     ::"r"(smem_u32(bar)), "r"((uint32_t)lead) : "memory");
    else
        asm volatile("{\n\t.reg .pred q;\n\tsetp.ne.u32 q, %2, 0;\n\t"
                     "@q tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;\n\t}"
                     ::"r"(smem_u32(bar)), "h"((uint16_t)3), "r"((uint32_t)lead) : "memory");
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

__device__ __forceinline__ void tc_ld16(uint32_t tmem, uint32_t (&r)[16])
{
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]),
          "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
        : "r"(tmem));
}
__device__ __forceinline__ uint32_t tc_ld1(uint32_t tmem)
{
    uint32_t r;
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x1.b32 {%0}, [%1];" : "=r"(r) : "r"(tmem));
    tc_wait_ld();
    return r;
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

// ------------------------------------------------------------------ 16-bit operands
// kind::f16 -> binary32.  `mn`: B is stored with its N dimension contiguous (keys as rows of a [keys x dims] B)
__host__ __device__ constexpr uint32_t tc_idesc_f16(bool bf16, int m, int n, bool mn)
{
    return (1u << 4) | ((bf16 ? 1u : 0u) << 7) | ((bf16 ? 1u : 0u) << 10) | ((mn ? 1u : 0u) << 16) | ((uint32_t)(n >> 3) << 17) |
           ((uint32_t)(m >> 4) << 24);
}
// B with N contiguous: blocks of 64 elements of N (a swizzled row of 128 bytes), `block` bytes from one to the next;
// eight rows (of K) make 1024 bytes
__device__ __forceinline__ uint32_t tc_desc_mn(uint32_t smem, uint32_t block) { return ((smem >> 4) & 0x3fff) | (((block >> 4) & 0x3fff) << 16); }
// A in TMEM (two 16-bit elements of K per column), B in shared memory
__device__ __forceinline__ void tc_mma_f16_ta(uint32_t d, uint32_t a, uint32_t b, uint32_t idesc, bool add, bool lead)
{
    asm volatile("{\n\t.reg .pred p, q;\n\t.reg .b64 db;\n\tsetp.ne.u32 p, %4, 0;\n\tsetp.ne.u32 q, %6, 0;\n\tmov.b64 db, {%2, %5};\n\t"
                 "@q tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], db, %3, p;\n\t}"
                 ::"r"(d), "r"(a), "r"(b), "r"(idesc), "r"((uint32_t)add), "r"(kTcDescHi), "r"((uint32_t)lead) : "memory");
}
// both in shared memory, K-major
__device__ __forceinline__ void tc_mma_f16_ss(uint32_t d, uint32_t a, uint32_t b, uint32_t idesc, bool add, bool lead)
{
    asm volatile("{\n\t.reg .pred p, q;\n\t.reg .b64 da, db;\n\tsetp.ne.u32 p, %4, 0;\n\tsetp.ne.u32 q, %6, 0;\n\t"
                 "mov.b64 da, {%1, %5};\n\tmov.b64 db, {%2, %5};\n\t"
                 "@q tcgen05.mma.cta_group::1.kind::f16 [%0], da, db, %3, p;\n\t}"
                 ::"r"(d), "r"(a), "r"(b), "r"(idesc), "r"((uint32_t)add), "r"(kTcDescHi), "r"((uint32_t)lead) : "memory");
}
__device__ __forceinline__ void tc_st32(uint32_t tmem, const uint32_t *r)
{
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x32.b32 [%32], "
        "{%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31};"
        ::"r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]),
          "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(r[16]), "r"(r[17]), "r"(r[18]), "r"(r[19]), "r"(r[20]),
          "r"(r[21]), "r"(r[22]), "r"(r[23]), "r"(r[24]), "r"(r[25]), "r"(r[26]), "r"(r[27]), "r"(r[28]), "r"(r[29]), "r"(r[30]),
          "r"(r[31]), "r"(tmem) : "memory");
}
__device__ __forceinline__ void tc_st16(uint32_t tmem, const uint32_t *r)
{
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x16.b32 [%16], {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15};"
        ::"r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]),
          "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(tmem) : "memory");
}
__device__ __forceinline__ void tc_wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
// 3-D box global -> shared memory of this CTA
__device__ __forceinline__ void tma_load3(uint32_t dst, const CUtensorMap *map, int x, int y, int z, uint32_t bar)
{
    asm volatile("cp.async.bulk.tensor.3d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];"
                 ::"r"(dst), "l"(map), "r"(x), "r"(y), "r"(z), "r"(bar) : "memory");
}
// 4-D box global -> shared memory of this CTA
__device__ __forceinline__ void tma_load4(uint32_t dst, const CUtensorMap *map, int x, int y, int z, int w, uint32_t bar)
{
    asm volatile("cp.async.bulk.tensor.4d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5}], [%6];"
                 ::"r"(dst), "l"(map), "r"(x), "r"(y), "r"(z), "r"(w), "r"(bar) : "memory");
}

}  // namespace aweq
