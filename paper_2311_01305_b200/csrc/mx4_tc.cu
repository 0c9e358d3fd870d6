// aweq_linear_mx4 on the tensor cores: tcgen05.mma on 4-bit elements with block scales, over TMA-fed tiles.
//   out[n,o] = sx_n sw_o sum_blocks a b sum (e2m1 x e2m1) + bias_o
// The products and block scales are multiplied and added by the tensor cores in binary32; steps and bias follow in binary32.
#include <math.h>

#include "mx4.cuh"
#include "tensorcore.cuh"

namespace aweq {

constexpr int kM4Block = 128;                  // bytes of K per stage: one swizzled row, 256 elements

struct alignas(8) Mx4Col { float step, bias; };
__device__ __forceinline__ Mx4Col mx4_col(const Mx4LinearArgs &p, long long o)
{
    Mx4Col c = {0.0f, 0.0f};
    if (o < p.O) {
        c.step = p.w_step ? p.w_step[o] : 1.0f;
        if (p.bias) c.bias = p.bias[o];
    }
    return c;
}

// ------------------------------------------------------------------ many tokens
// Output tiles of 256 tokens x 256 channels, each by a pair of CTAs (cta_group::2): a CTA stages its 128 tokens, half of the
// weights, its tokens' scales and all of the channels' scales.  Persistent: a pair takes every (pairs)-th tile.
//
// TMEM: 512 columns do not hold two accumulators of 256 and the scales.  The two overlap by 96 columns, which the epilogue takes
// out first: then the next tile's products may start.  Scales have 96 columns, two buffers (E4M3) or four, since a copy into TMEM is
// not in order with the products before it: the buffer's last products are waited for (that many stages back, so the pipe stays fed).
// Warps: 0 copies, 1 issues the products (in the pair's even CTA), 4-11 write the output, two to a quarter of the TMEM lanes.
// 4099 x 5120 x 13824 in blocks of 32: 110-120 us by itself, 4.8-5.3 PFLOP/s (3.1 to 3.4 of the measured bf16
// rates; nominal is 4), 130 in a row at the power cap.  A stage of 256 columns takes some 690 cycles for 512 of products: the tensor pipe is 70 % busy, the L2
// sends every SM some 55 bytes a cycle, near its limit; larger tiles do not fit TMEM beside the scales.  Scales' copies by a warp of their own: 127 us.
constexpr int kM4BigStages = 5, kM4BigThreads = 384, kM4Overlap = 96, kM4ScaleCols = 96;
constexpr int kM4SecondAcc = 256 - kM4Overlap, kM4Scales = 512 - kM4ScaleCols;
constexpr int kM4OutPitch = 80;                // bytes of a staged output row: 32 columns and 16 bytes against bank conflicts
static_assert(kM4SecondAcc + 256 <= kM4Scales, "columns of TMEM");
__host__ __device__ constexpr int m4_big_stage(int fmt) { return 2 * 128 * kM4Block + 3 * mx4_group_tiles(fmt) * kMx4Tile; }
struct M4BigShared {
    uint64_t full[kM4BigStages], empty[kM4BigStages], acc_full[2], acc_free;
    uint32_t tmem;
    Mx4Col col[256];
    alignas(16) unsigned char out[8][32 * kM4OutPitch];
};
__host__ __device__ constexpr size_t m4_big_smem(int fmt) { return 1024 + (size_t)kM4BigStages * m4_big_stage(fmt) + sizeof(M4BigShared); }
static_assert(m4_big_smem(AWEQ_MX4_E4M3) <= 227 * 1024, "shared memory of a CTA");

__device__ __forceinline__ void m4_big_tile(long long t, int mt, int nt, int *m, int *n)
{
    // eight row blocks at a time, so that the tiles in flight share both operands in the L2
    const long long group = 8ll * nt;
    const int g = (int)(t / group), first = g * 8, height = min(8, mt - first), r = (int)(t % group);
    *m = first + r % height;
    *n = r / height;
}

template <class D, int FMT>
__global__ void __launch_bounds__(kM4BigThreads, 1)
mx4_big_kernel(const Mx4LinearArgs p, const __grid_constant__ CUtensorMap mapX, const __grid_constant__ CUtensorMap mapW,
               const __grid_constant__ CUtensorMap mapSx, const __grid_constant__ CUtensorMap mapSw, int mt, int nt, int vec_out)
{
    constexpr int T = mx4_group_tiles(FMT), kStage = m4_big_stage(FMT), kScaleAt = 2 * 128 * kM4Block, kBufs = kM4ScaleCols / (12 * T);
    constexpr bool E8M0 = FMT == AWEQ_MX4_E8M0;
    extern __shared__ unsigned char raw[];
    unsigned char *stages = reinterpret_cast<unsigned char *>((reinterpret_cast<uintptr_t>(raw) + 1023) & ~(uintptr_t)1023);
    M4BigShared &sh = *reinterpret_cast<M4BigShared *>(stages + kM4BigStages * kStage);
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const uint32_t rank = cluster_ctarank();
    const int nkb = (p.K + 255) / 256;
    const long long tiles = (long long)mt * nt, step = gridDim.x / 2;
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    if (threadIdx.x == 0) {
        for (int s = 0; s < kM4BigStages; ++s) {
            mbar_init(&sh.full[s], 1);
            mbar_init(&sh.empty[s], 1);
        }
        mbar_init(&sh.acc_full[0], 1);
        mbar_init(&sh.acc_full[1], 1);
        mbar_init(&sh.acc_free, 16);
        mbar_init_fence();
        tma_prefetch_map(&mapX);
        tma_prefetch_map(&mapW);
        tma_prefetch_map(&mapSx);
        tma_prefetch_map(&mapSw);
    }
    if (warp == 1) tc_alloc<2>(&sh.tmem, 512);
    tc_fence_before();
    __syncthreads();
    cluster_sync_all();
    tc_fence_after();
    const uint32_t tmem = sh.tmem;
    asm volatile("griddepcontrol.wait;" ::: "memory");

    bool ok = true;
    if (warp == 0) {
        if (lane == 0) {
            int s = 0;
            uint32_t ph = 0;
            for (long long t = blockIdx.x / 2; ok && t < tiles; t += step) {
                int m, n;
                m4_big_tile(t, mt, nt, &m, &n);
                const int row = m * 256 + (int)rank * 128, col = n * 256 + (int)rank * 128;
                // (tiles of scales: nkb groups of T to a block of 128 rows)
                int sx = (m * 2 + (int)rank) * nkb * T, sw = n * 2 * nkb * T;
                for (int kb = 0; kb < nkb; ++kb, sx += T, sw += T) {
                    if (!mbar_wait_cluster(&sh.empty[s], ph ^ 1)) { ok = false; break; }
                    const uint32_t bar = cluster_map(&sh.full[s], 0), dst = smem_u32(stages + s * kStage);
                    if (rank == 0) mbar_arrive_expect_tx(&sh.full[s], 2 * kStage);
                    tma_load2<2>(dst, &mapX, kb * kM4Block, row, bar);
                    tma_load2<2>(dst + 128 * kM4Block, &mapW, kb * kM4Block, col, bar);
                    tma_load2<2>(dst + kScaleAt, &mapSx, 0, sx, bar);
                    tma_load2<2>(dst + kScaleAt + T * kMx4Tile, &mapSw, 0, sw, bar);
                    tma_load2<2>(dst + kScaleAt + 2 * T * kMx4Tile, &mapSw, 0, sw + nkb * T, bar);
                    if (++s == kM4BigStages) { s = 0; ph ^= 1; }
                }
            }
            if (!ok && rank == 0)              // gave up: let what is under way land (bounded) before the memory goes
                for (int i = 0; i < kM4BigStages; ++i) mbar_wait(&sh.full[i], ph ^ (i >= s ? 1u : 0u));
        }
    } else if (warp == 1) {
        if (rank == 0) {
            const bool lead = tc_elect();
            int s = 0, back = kM4BigStages - kBufs, it = 0;
            uint32_t ph = 0, back_ph = 1, buf = 0;
            const uint32_t idesc = tc_idesc_mx4(E8M0, 256, 256);
            for (long long t = blockIdx.x / 2; ok && t < tiles; t += step, ++it) {
                const uint32_t acc = tmem + (it & 1 ? kM4SecondAcc : 0);
                if (it > 0 && !mbar_wait_cluster(&sh.acc_free, (it - 1) & 1)) { ok = false; break; }
                tc_fence_after();
                for (int kb = 0; kb < nkb; ++kb) {
                    // the products that read this buffer of scales (at the start: a phase that counts as over)
                    if (!mbar_wait_cluster(&sh.full[s], ph) || !mbar_wait_cluster(&sh.empty[back], back_ph)) { ok = false; break; }
                    tc_fence_after();
                    const uint32_t a = smem_u32(stages + s * kStage), sf = tmem + kM4Scales + buf * (12 * T);
                    const uint32_t da = tc_desc(a), db = tc_desc(a + 128 * kM4Block);
#pragma unroll
                    for (int i = 0; i < T; ++i) {
                        tc_copy_scales<2>(sf + i * 4, a + kScaleAt + i * kMx4Tile, lead);
                        tc_copy_scales<2>(sf + T * 4 + i * 8, a + kScaleAt + (T + i) * kMx4Tile, lead);
                        tc_copy_scales<2>(sf + T * 4 + i * 8 + 4, a + kScaleAt + (2 * T + i) * kMx4Tile, lead);
                    }
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        const int i = E8M0 ? k >> 1 : k;
                        tc_mma_mx4<2, E8M0>(acc, da + 2 * k, db + 2 * k, E8M0 ? tc_idesc_mx4_half(idesc, k & 1) : idesc, sf + i * 4,
                                            sf + T * 4 + i * 8, (kb | k) != 0, lead);
                    }
                    tc_commit<2>(&sh.empty[s], lead);
                    if (++s == kM4BigStages) { s = 0; ph ^= 1; }
                    if (++back == kM4BigStages) { back = 0; back_ph ^= 1; }
                    buf = (buf + 1) % kBufs;
                }
                if (ok) tc_commit<2>(&sh.acc_full[it & 1], lead);
            }
        }
    } else if (warp >= 4) {
        const int q = warp & 3, half = (warp - 4) >> 2, tid = threadIdx.x - 128;
        unsigned char *buf = sh.out[warp - 4];
        int it = 0;
        for (long long t = blockIdx.x / 2; t < tiles; t += step, ++it) {
            int m, n;
            m4_big_tile(t, mt, nt, &m, &n);
            const long long row0 = (long long)m * 256 + rank * 128 + q * 32, row = row0 + lane, o0 = (long long)n * 256;
            named_bar_sync(1, 256);
            sh.col[tid] = mx4_col(p, o0 + tid);
            const float sx = row < p.N && p.x_step ? p.x_step[row] : 1.0f;
            named_bar_sync(1, 256);
            const bool got = mbar_wait_cluster(&sh.acc_full[it & 1], (it >> 1) & 1);
            if (!named_bar_and(2, 256, got)) { ok = false; break; }
            tc_fence_after();
            const uint32_t at = tmem + (it & 1 ? kM4SecondAcc : 0) + ((uint32_t)(q * 32) << 16);
            // the three chunks of 32 columns that the next accumulator overlaps first, one to half 0 and two to half 1
            const int first = it & 1 ? 0 : 5, rest = it & 1 ? 3 : 0;
            uint32_t S[2][32];
            tc_ld32(at + (first + half) * 32, S[0]);
            if (half) tc_ld32(at + (first + 2) * 32, S[1]);
            tc_wait_ld();
            tc_fence_before();
            __syncwarp();
            if (lane == 0) cluster_mbar_arrive(cluster_map(&sh.acc_free, 0));
            auto write = [&](const uint32_t (&x)[32], int c0) {
                if (row0 >= p.N || o0 + c0 >= p.O) return;
                uint32_t packed[16];
#pragma unroll
                for (int j = 0; j < 32; j += 2) {
                    const Mx4Col c = sh.col[c0 + j], d = sh.col[c0 + j + 1];
                    packed[j / 2] = D::encode2(__fmaf_rn(__uint_as_float(x[j]) * sx, c.step, c.bias),
                                               __fmaf_rn(__uint_as_float(x[j + 1]) * sx, d.step, d.bias));
                }
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    *reinterpret_cast<uint4 *>(buf + lane * kM4OutPitch + j * 16) =
                        make_uint4(packed[4 * j], packed[4 * j + 1], packed[4 * j + 2], packed[4 * j + 3]);
                __syncwarp();
                const int cols = (int)min(32ll, p.O - (o0 + c0));
                if (vec_out && cols % 8 == 0) {
                    // eight rows of 64 bytes per store
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const int r = i * 8 + (lane >> 2), c = (lane & 3) * 8;
                        if (row0 + r < p.N && c < cols)
                            *reinterpret_cast<uint4 *>(p.out + (row0 + r) * p.ldo + o0 + c0 + c) =
                                *reinterpret_cast<const uint4 *>(buf + r * kM4OutPitch + c * 2);
                    }
                } else {
                    for (int r = 0; r < 32 && row0 + r < p.N; ++r)
                        if (lane < cols) p.out[(row0 + r) * p.ldo + o0 + c0 + lane] = *reinterpret_cast<const uint16_t *>(buf + r * kM4OutPitch + lane * 2);
                }
                __syncwarp();
            };
            write(S[0], (first + half) * 32);
            if (half) write(S[1], (first + 2) * 32);
            // the other five: three and two
#pragma unroll 1
            for (int c = rest + (half ? 3 : 0); c < rest + (half ? 5 : 3); ++c) {
                tc_ld32(at + c * 32, S[0]);
                tc_wait_ld();
                write(S[0], c * 32);
            }
            tc_fence_before();
        }
    }
    if (!ok && p.st) atomicAdd(&p.st->wait_timeout, 1ull);
    tc_fence_before();
    __syncthreads();
    cluster_sync_all();
    if (warp == 1) tc_dealloc<2>(tmem, 512);
}

template <class D, int FMT>
static aweq_status m4_big_launch(const Mx4LinearArgs &a, cudaStream_t stream)
{
    constexpr int T = mx4_group_tiles(FMT);
    CUtensorMap mx, mw, sx, sw;
    const long long per_row = mx4_row_tiles(a.K, FMT);
    aweq_status rc = tma_bytes_map(&mx, a.X, a.N, a.K / 2, a.K / 2, 128);
    if (rc == AWEQ_OK) rc = tma_bytes_map(&mw, a.W, a.O, a.K / 2, a.K / 2, 128);
    if (rc == AWEQ_OK) rc = tma_tiles_map(&sx, a.x_scales, (a.N + 127) / 128 * per_row, T);
    if (rc == AWEQ_OK) rc = tma_tiles_map(&sw, a.w_scales, (a.O + 127) / 128 * per_row, T);
    if (rc != AWEQ_OK) return rc;
    static std::atomic<unsigned long long> allowed{0};
    AWEQ_CUDA_OK(allow_smem(mx4_big_kernel<D, FMT>, m4_big_smem(FMT), allowed));
    const int mt = (int)((a.N + 255) / 256), nt = (a.O + 255) / 256;
    const long long tiles = (long long)mt * nt;
    const unsigned pairs = (unsigned)(tiles < kSmCount / 2 ? tiles : kSmCount / 2);
    const int vec = (a.ldo % 8 == 0) && ((reinterpret_cast<uintptr_t>(a.out) & 15) == 0);
    const cudaError_t e = launch_pdl_cluster(mx4_big_kernel<D, FMT>, dim3(pairs * 2), dim3(kM4BigThreads), m4_big_smem(FMT), stream, 2, a,
                                             mx, mw, sx, sw, mt, nt, vec);
    note_launch();
    return e == cudaSuccess ? AWEQ_OK : cuda_failed(e);
}

// ------------------------------------------------------------------ few tokens
// The layer is bound by the weights here.  The weights are the 128-row operand and the tokens, up to 128, the other: a product costs
// what the tokens there are ask for, and reads nothing that is not there.  Where few channels leave SMs idle, K is cut over the
// CTAs of a cluster, whose sums are added through distributed shared memory in the order of the slices.  A CTA's ring takes as much of an SM
// as its blocks of K fill: with few of them two or three CTAs share one.  Warps: 0 copies, 1 issues the products; all write the output.
// 24 x 4096 x 12288 in blocks of 16, weights from memory: 11.3 us, 2.5 TB/s (a copy of as many bytes 4.4 us and a launch's start and end);
// with the weights in the L2 8.6.  1 x 768 x 768: 5.7 us from memory, 2.9 from the L2: latency.
constexpr int kM4SplitMaxStages = 8;
struct M4SplitPlan {
    int bn, slices, stages;                    // tokens, as a multiple of 16 up to 128, slices of K, ring
    int stage_bytes, scale_cols, cols;         // TMEM: a buffer of scales, all
};
struct M4SplitShared {
    uint64_t full[kM4SplitMaxStages], empty[kM4SplitMaxStages], acc_full;
    uint32_t tmem;
};

template <class D, int FMT>
__global__ void __launch_bounds__(256)
mx4_split_kernel(const Mx4LinearArgs p, const __grid_constant__ CUtensorMap mapX, const __grid_constant__ CUtensorMap mapW,
                 const M4SplitPlan plan, int vec_out)
{
    constexpr int T = mx4_group_tiles(FMT);
    constexpr bool E8M0 = FMT == AWEQ_MX4_E8M0;
    extern __shared__ unsigned char raw[];
    __shared__ M4SplitShared sh;
    unsigned char *stages = reinterpret_cast<unsigned char *>((reinterpret_cast<uintptr_t>(raw) + 1023) & ~(uintptr_t)1023);
    float *part = reinterpret_cast<float *>(stages);
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int bn = plan.bn, x_at = 128 * kM4Block, sf_at = x_at + bn * kM4Block;
    const int slices = plan.slices, slice = blockIdx.x;
    const int nkb = (p.K + 255) / 256;
    const int kb0 = (int)((long long)nkb * slice / slices), kb1 = (int)((long long)nkb * (slice + 1) / slices);
    const int rows = (int)p.N;
    const int o0 = blockIdx.y * 128;
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    if (threadIdx.x == 0) {
        for (int s = 0; s < plan.stages; ++s) {
            mbar_init(&sh.full[s], 1);
            mbar_init(&sh.empty[s], 1);
        }
        mbar_init(&sh.acc_full, 1);
        mbar_init_fence();
        tma_prefetch_map(&mapX);
        tma_prefetch_map(&mapW);
    }
    if (warp == 1) tc_alloc<1>(&sh.tmem, (uint32_t)plan.cols);
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = sh.tmem;
    asm volatile("griddepcontrol.wait;" ::: "memory");

    bool ok = true;
    if (warp == 0) {
        if (lane == 0) {
            int s = 0;
            uint32_t ph = 0;
            const unsigned char *sw = p.w_scales + ((long long)blockIdx.y * mx4_row_tiles(p.K, FMT) + (long long)kb0 * T) * kMx4Tile;
            const unsigned char *sx = p.x_scales + (long long)kb0 * T * kMx4Tile;
            const uint32_t bytes = 128 * kM4Block + bn * kM4Block + 2 * T * kMx4Tile;
            for (int kb = kb0; kb < kb1; ++kb, sw += T * kMx4Tile, sx += T * kMx4Tile) {
                if (!mbar_wait(&sh.empty[s], ph ^ 1)) { ok = false; break; }
                unsigned char *const st = stages + s * plan.stage_bytes;
                const uint32_t bar = smem_u32(&sh.full[s]), dst = smem_u32(st);
                mbar_arrive_expect_tx(&sh.full[s], bytes);
                tma_load2<1>(dst, &mapW, kb * kM4Block, o0, bar);
                bulk_g2s(st + sf_at, sw, T * kMx4Tile, &sh.full[s]);
                tma_load2<1>(dst + x_at, &mapX, kb * kM4Block, 0, bar);
                bulk_g2s(st + sf_at + T * kMx4Tile, sx, T * kMx4Tile, &sh.full[s]);
                if (++s == plan.stages) { s = 0; ph ^= 1; }
            }
            if (!ok)                           // gave up: let what is under way land (bounded) before the memory goes
                for (int i = 0; i < plan.stages; ++i) mbar_wait(&sh.full[i], ph ^ (i >= s ? 1u : 0u));
        }
    } else if (warp == 1) {
        const bool lead = tc_elect();
        int s = 0, back = plan.stages - 2;
        uint32_t ph = 0, back_ph = 1, buf = 0;
        const uint32_t idesc = tc_idesc_mx4(E8M0, 128, bn);
        for (int kb = kb0; kb < kb1; ++kb) {
            if (!mbar_wait(&sh.full[s], ph) || !mbar_wait(&sh.empty[back], back_ph)) { ok = false; break; }
            tc_fence_after();
            const uint32_t a = smem_u32(stages + s * plan.stage_bytes), sf = tmem + bn + buf * plan.scale_cols;
            const uint32_t da = tc_desc(a), db = tc_desc(a + x_at), xs = sf + T * 4;
#pragma unroll
            for (int i = 0; i < T; ++i) {
                tc_copy_scales<1>(sf + i * 4, a + sf_at + i * kMx4Tile, lead);
                tc_copy_scales<1>(xs + i * 4, a + sf_at + (T + i) * kMx4Tile, lead);
            }
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const int i = E8M0 ? k >> 1 : k;
                tc_mma_mx4<1, E8M0>(tmem, da + 2 * k, db + 2 * k, E8M0 ? tc_idesc_mx4_half(idesc, k & 1) : idesc, sf + i * 4,
                                    xs + i * 4, kb > kb0 || k > 0, lead);
            }
            tc_commit<1>(&sh.empty[s], lead);
            if (++s == plan.stages) { s = 0; ph ^= 1; }
            if (++back == plan.stages) { back = 0; back_ph ^= 1; }
            buf ^= 1;
        }
        if (ok) {
            tc_commit<1>(&sh.acc_full, lead);
            ok = mbar_wait(&sh.acc_full, 0);
        }
    }
    if (!ok && p.st) atomicAdd(&p.st->wait_timeout, 1ull);
    __syncthreads();                           // every product and copy of this CTA is done (or has been given up)
    tc_fence_after();
    constexpr int pitch = 132;                 // floats of a token's row of 128 channels
    {
        // a lane holds a channel: the four quarters of TMEM by warp % 4, 16 tokens at a time by the halves of the CTA
        const int q = warp & 3;
        for (int c = (warp >> 2) * 16; c < bn; c += 32) {
            uint32_t S[16];
            tc_ld16(tmem + c + ((uint32_t)(q * 32) << 16), S);
            tc_wait_ld();
#pragma unroll
            for (int j = 0; j < 16; ++j)
                if (c + j < rows) part[(c + j) * pitch + q * 32 + lane] = __uint_as_float(S[j]);
        }
    }
    tc_fence_before();
    if (slices > 1) cluster_sync_all();
    else __syncthreads();
    if (warp == 1) {
        __syncwarp();
        tc_fence_after();
        tc_dealloc<1>(tmem, (uint32_t)plan.cols);
    }
    // tokens slice, slice + slices, ... are this CTA's: a warp per token, four channels a lane
    const int c = lane * 4;
    Mx4Col col[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) col[j] = mx4_col(p, o0 + c + j);
    for (int r = slice + slices * warp; r < rows; r += slices * 8) {
        float4 v = make_float4(0, 0, 0, 0);
        for (int k = 0; k < slices; ++k) {
            float4 x;
            if (slices == 1) x = *reinterpret_cast<const float4 *>(part + r * pitch + c);
            else
                asm volatile("ld.shared::cluster.v4.f32 {%0,%1,%2,%3}, [%4];" : "=f"(x.x), "=f"(x.y), "=f"(x.z), "=f"(x.w)
                             : "r"(cluster_map(part + r * pitch + c, k)) : "memory");
            v.x += x.x; v.y += x.y; v.z += x.z; v.w += x.w;
        }
        const float sx = p.x_step ? p.x_step[r] : 1.0f;
        const float y[4] = {__fmaf_rn(v.x * sx, col[0].step, col[0].bias), __fmaf_rn(v.y * sx, col[1].step, col[1].bias),
                            __fmaf_rn(v.z * sx, col[2].step, col[2].bias), __fmaf_rn(v.w * sx, col[3].step, col[3].bias)};
        uint16_t *dst = p.out + r * p.ldo + o0 + c;
        if (vec_out && o0 + c + 4 <= p.O)
            *reinterpret_cast<uint2 *>(dst) = make_uint2(D::encode2(y[0], y[1]), D::encode2(y[2], y[3]));
        else
#pragma unroll
            for (int j = 0; j < 4; ++j)
                if (o0 + c + j < p.O) dst[j] = D::encode(y[j]);
    }
    if (slices > 1) cluster_sync_all();        // nobody leaves while its sums may still be read
}

constexpr int kM4SplitMaxSmem = 216 * 1024;

template <class D, int FMT>
static aweq_status m4_split_launch(const Mx4LinearArgs &a, int slices, cudaStream_t stream)
{
    constexpr int T = mx4_group_tiles(FMT);
    M4SplitPlan s;
    s.bn = (int)((a.N + 15) / 16 * 16);
    s.slices = slices;
    s.stage_bytes = (128 + s.bn) * kM4Block + 2 * T * kMx4Tile;
    s.stage_bytes = (s.stage_bytes + 1023) / 1024 * 1024;
    s.scale_cols = T * 8;
    s.cols = 32;
    while (s.cols < s.bn + 2 * s.scale_cols) s.cols *= 2;
    // (no more stages than a slice has blocks: 16 x 4096 x 4096 in four slices 5.0 us, with eight stages 5.5)
    const int out_bytes = s.bn * 132 * 4, blocks = ((a.K + 255) / 256 + slices - 1) / slices;
    s.stages = kM4SplitMaxSmem / s.stage_bytes;
    if (s.stages > kM4SplitMaxStages) s.stages = kM4SplitMaxStages;
    if (s.stages > blocks) s.stages = blocks;
    if (s.stages < 3) s.stages = 3;
    int smem = s.stages * s.stage_bytes;
    if (smem < out_bytes) smem = out_bytes;
    smem += 1024;
    CUtensorMap mx, mw;
    aweq_status rc = tma_bytes_map(&mx, a.X, a.N, a.K / 2, a.K / 2, s.bn);
    if (rc == AWEQ_OK) rc = tma_bytes_map(&mw, a.W, a.O, a.K / 2, a.K / 2, 128);
    if (rc != AWEQ_OK) return rc;
    static std::atomic<unsigned long long> allowed{0};
    AWEQ_CUDA_OK(allow_smem(mx4_split_kernel<D, FMT>, 226 * 1024, allowed));
    const dim3 grid((unsigned)slices, (unsigned)((a.O + 127) / 128));
    const int vec = (a.ldo % 4 == 0) && ((reinterpret_cast<uintptr_t>(a.out) & 7) == 0);
    const cudaError_t e = launch_pdl_cluster(mx4_split_kernel<D, FMT>, grid, dim3(256), (size_t)smem, stream, (unsigned)slices, a, mx, mw, s, vec);
    note_launch();
    return e == cudaSuccess ? AWEQ_OK : cuda_failed(e);
}

// Which kernel, and into how many slices of K.  Measured on the device, in microseconds (weights in the L2):
//   16 x 4096 x 4096   1 to 4 slices 7.2, 5.5, 5.1, 5.0 (32 to 128 CTAs), 5 and 8 slices 8.2, 9.7 (more CTAs than SMs); pairs 9.7
//   16 x 13824 x 5120  1 to 4 slices 19.3, 12.3, 11.0, 18.1 (40 to 160 CTAs); pairs 24.1
//   24 x 4096 x 12288  1 slice 8.6 (96 CTAs), 2 slices 12.0; pairs 13.8         1 x 768 x 768  1 to 3 slices 2.9, 3.4, 3.4; pairs 5.6
//   64 x 5120 x 13824  1 slice 11.5; pairs 13.7        128 x 4096 x 4096  4 slices 8.5; pairs 11.1
//   128 x 5120 x 13824 1 slice 16.8; pairs 15.1        256 x 4096 x 4096  4 slices 13.0; pairs 11.2
// So: as many slices as leave every CTA an SM of its own and two blocks of K; pairs beyond 128 tokens, and beyond 64 where the channels
// alone fill the SMs.
template <class D, int FMT>
static aweq_status m4_choose(const Mx4LinearArgs &a, cudaStream_t stream)
{
    const int nkb = (a.K + 255) / 256;
    const long long ct = (a.O + 127) / 128;                      // (channels lie on the grid's second dimension)
    if (a.N > 128 || (a.N > 64 && 2 * ct > kSmCount) || ct > 65535) return m4_big_launch<D, FMT>(a, stream);
    int slices = 1;
    while (slices < 4 && 2 * (slices + 1) <= nkb && ct * (slices + 1) <= kSmCount) ++slices;
    return m4_split_launch<D, FMT>(a, slices, stream);
}

aweq_status run_linear_mx4(const Mx4LinearArgs &a, aweq_dtype dt, cudaStream_t stream)
{
    if (dt == AWEQ_F16) return a.fmt == AWEQ_MX4_E8M0 ? m4_choose<F16, AWEQ_MX4_E8M0>(a, stream) : m4_choose<F16, AWEQ_MX4_E4M3>(a, stream);
    return a.fmt == AWEQ_MX4_E8M0 ? m4_choose<BF16, AWEQ_MX4_E8M0>(a, stream) : m4_choose<BF16, AWEQ_MX4_E4M3>(a, stream);
}

}  // namespace aweq
