// aweq_linear_w8a8 on the tensor cores: tcgen05.mma kind::i8 over TMA-fed tiles.
#include "linear8.cuh"
#include "tensorcore.cuh"

namespace aweq {

aweq_status tma_bytes_map(CUtensorMap *map, const void *base, long long rows, long long cols, long long ld, int box_rows)
{
    using Encode = CUresult (*)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *, const cuuint64_t *,
                                const cuuint32_t *, const cuuint32_t *, CUtensorMapInterleave, CUtensorMapSwizzle,
                                CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
    static const Encode encode = [] {
        void *f = nullptr;
        cudaDriverEntryPointQueryResult found = cudaDriverEntryPointSymbolNotFound;
        if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &f, 12000, cudaEnableDefault, &found) != cudaSuccess ||
            found != cudaDriverEntryPointSuccess)
            f = nullptr;
        return reinterpret_cast<Encode>(f);
    }();
    if (!encode) return AWEQ_ERR_UNSUPPORTED;
    const cuuint64_t dims[2] = {(cuuint64_t)cols, (cuuint64_t)rows}, pitch[1] = {(cuuint64_t)ld};
    const cuuint32_t box[2] = {128, (cuuint32_t)box_rows}, step[2] = {1, 1};
    const CUresult r = encode(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, const_cast<void *>(base), dims, pitch, box, step,
                              CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                              CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    return r == CUDA_SUCCESS ? AWEQ_OK : cuda_failed(cudaErrorInvalidValue);
}

constexpr int kL8Block = 128;                  // bytes of K per stage: one swizzled row

// sum of the 128 code bytes of a staged row.  A row's 16-byte pieces are permuted by the swizzle, which a
// sum does not see; the lanes start at different pieces so that they spread over the banks.
__device__ __forceinline__ uint32_t staged_row_sum(const unsigned char *row, int lane)
{
    uint32_t s = 0;
#pragma unroll
    for (int c = 0; c < 8; ++c) {
        const uint4 v = *reinterpret_cast<const uint4 *>(row + ((c + lane) & 7) * 16);
        s = __dp4a(v.x, 0x01010101u, s);
        s = __dp4a(v.y, 0x01010101u, s);
        s = __dp4a(v.z, 0x01010101u, s);
        s = __dp4a(v.w, 0x01010101u, s);
    }
    return s;
}

struct alignas(16) Linear8Col {
    float step, bias;
    int zp;
    uint32_t sum;
};
__device__ __forceinline__ Linear8Col linear8_col(const Linear8Args &p, long long o)
{
    Linear8Col c = {0.0f, 0.0f, 0, 0u};
    if (o < p.O) {
        c.step = __ldg(p.w_step + o * p.w_inc);
        c.zp = __ldg(p.w_zp + o * p.w_inc);
        c.sum = (uint32_t)__ldg(p.w_sum + o);
        if (p.bias) c.bias = __ldg(p.bias + o);
    }
    return c;
}

// ------------------------------------------------------------------ many tokens
// 256 x 256 output tiles, each by a pair of CTAs (cta_group::2): a CTA stages its 128 tokens and half of
// the 256 channels, and holds the 128 x 256 sums of its tokens in TMEM, twice, so that the
// epilogue of one tile runs under the products of the next.  Persistent: a pair takes every
// (pairs)-th tile.  Warps: 0 copies, 1 issues the products (in the pair's even CTA), 2-3 add up the
// tokens' codes from the stages (after the products have used them: that completion is the one
// signal both CTAs get), 4-7 write the output.
constexpr int kBigStages = 6;
constexpr int kBigStageBytes = 2 * 128 * kL8Block;
constexpr int kBigOutPitch = 144;              // bytes of a staged output row: 64 columns and 16 bytes against bank conflicts
struct BigShared {
    uint64_t full[kBigStages], done[kBigStages], empty[kBigStages], acc_full[2], acc_empty[2], rx_full[2], rx_empty[2];
    uint32_t tmem;
    float reach[4];
    uint32_t rx[2][128];
    Linear8Col col[256];
    alignas(16) unsigned char out[4][32 * kBigOutPitch];
};
constexpr size_t kBigSmem = 1024 + (size_t)kBigStages * kBigStageBytes + sizeof(BigShared);

__device__ __forceinline__ void big_tile(long long t, int mt, int nt, int *m, int *n)
{
    // eight row blocks at a time, so that the tiles in flight share both operands in the L2
    const long long group = 8ll * nt;
    const int g = (int)(t / group), first = g * 8, height = min(8, mt - first), r = (int)(t % group);
    *m = first + r % height;
    *n = r / height;
}

template <class D>
__global__ void __launch_bounds__(256, 1)
linear8_big_kernel(const Linear8Args p, const __grid_constant__ CUtensorMap mapX, const __grid_constant__ CUtensorMap mapW,
                   int mt, int nt, int vec_out)
{
    extern __shared__ unsigned char raw[];
    unsigned char *stages = reinterpret_cast<unsigned char *>((reinterpret_cast<uintptr_t>(raw) + 1023) & ~(uintptr_t)1023);
    BigShared &sh = *reinterpret_cast<BigShared *>(stages + kBigStages * kBigStageBytes);
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const uint32_t rank = cluster_ctarank();
    const int nkb = (p.K + kL8Block - 1) / kL8Block;
    const long long tiles = (long long)mt * nt, step = gridDim.x / 2;
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    if (threadIdx.x == 0) {
        for (int s = 0; s < kBigStages; ++s) {
            mbar_init(&sh.full[s], 1);
            mbar_init(&sh.done[s], 1);
            mbar_init(&sh.empty[s], 2);
        }
        for (int a = 0; a < 2; ++a) {
            mbar_init(&sh.acc_full[a], 1);
            mbar_init(&sh.acc_empty[a], 8);
            mbar_init(&sh.rx_full[a], 2);
            mbar_init(&sh.rx_empty[a], 4);
        }
        mbar_init_fence();
        tma_prefetch_map(&mapX);
        tma_prefetch_map(&mapW);
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
                big_tile(t, mt, nt, &m, &n);
                const int row = m * 256 + (int)rank * 128, col = n * 256 + (int)rank * 128;
                for (int kb = 0; kb < nkb; ++kb) {
                    if (!mbar_wait(&sh.empty[s], ph ^ 1)) { ok = false; break; }
                    const uint32_t bar = cluster_map(&sh.full[s], 0), dst = smem_u32(stages + s * kBigStageBytes);
                    if (rank == 0) mbar_arrive_expect_tx(&sh.full[s], 2 * kBigStageBytes);
                    tma_load2<2>(dst, &mapX, kb * kL8Block, row, bar);
                    tma_load2<2>(dst + 128 * kL8Block, &mapW, kb * kL8Block, col, bar);
                    if (++s == kBigStages) { s = 0; ph ^= 1; }
                }
            }
            if (!ok && rank == 0)              // gave up: let what is under way land (bounded) before the memory goes
                for (int i = 0; i < kBigStages; ++i) mbar_wait(&sh.full[i], ph ^ (i >= s ? 1u : 0u));
        }
    } else if (warp == 1) {
        if (lane == 0 && rank == 0) {
            int s = 0, it = 0;
            uint32_t ph = 0;
            const uint32_t idesc = tc_idesc_u8(256, 256);
            for (long long t = blockIdx.x / 2; ok && t < tiles; t += step, ++it) {
                const int acc = it & 1;
                if (!mbar_wait_cluster(&sh.acc_empty[acc], ((it >> 1) & 1) ^ 1)) { ok = false; break; }
                tc_fence_after();
                for (int kb = 0; kb < nkb; ++kb) {
                    if (!mbar_wait_cluster(&sh.full[s], ph)) { ok = false; break; }
                    tc_fence_after();
                    const uint32_t a = smem_u32(stages + s * kBigStageBytes);
                    const uint64_t da = tc_desc(a), db = tc_desc(a + 128 * kL8Block);
#pragma unroll
                    for (int k = 0; k < 4; ++k)
                        tc_mma_u8<2>(tmem + acc * 256, da + 2 * k, db + 2 * k, idesc, (kb | k) != 0);
                    tc_commit<2>(&sh.done[s]);
                    if (++s == kBigStages) { s = 0; ph ^= 1; }
                }
                if (ok) tc_commit<2>(&sh.acc_full[acc]);
            }
        }
    } else if (warp < 4) {
        int s = 0, it = 0;
        uint32_t ph = 0;
        const int r0 = (warp - 2) * 64 + lane;
        for (long long t = blockIdx.x / 2; ok && t < tiles; t += step, ++it) {
            const int acc = it & 1;
            uint32_t a = 0, b = 0;
            for (int kb = 0; kb < nkb; ++kb) {
                ok = mbar_wait_cluster(&sh.done[s], ph);
                if (!__all_sync(0xffffffffu, ok)) { ok = false; break; }
                const unsigned char *x = stages + s * kBigStageBytes + r0 * kL8Block;
                a += staged_row_sum(x, lane);
                b += staged_row_sum(x + 32 * kL8Block, lane);
                __syncwarp();
                if (lane == 0) mbar_arrive(&sh.empty[s]);
                if (++s == kBigStages) { s = 0; ph ^= 1; }
            }
            if (!ok) break;
            ok = mbar_wait(&sh.rx_empty[acc], ((it >> 1) & 1) ^ 1);
            if (!__all_sync(0xffffffffu, ok)) { ok = false; break; }
            sh.rx[acc][r0] = a;
            sh.rx[acc][r0 + 32] = b;
            __syncwarp();
            if (lane == 0) mbar_arrive(&sh.rx_full[acc]);
        }
    } else {
        const int q = warp - 4, tid = threadIdx.x - 128;
        unsigned char *buf = sh.out[q];
        int it = 0;
        for (long long t = blockIdx.x / 2; t < tiles; t += step, ++it) {
            const int acc = it & 1;
            int m, n;
            big_tile(t, mt, nt, &m, &n);
            const long long row0 = (long long)m * 256 + rank * 128 + q * 32, row = row0 + lane, o0 = (long long)n * 256;
            // the channels' pairs, and the largest reach of their zero-points
            named_bar_sync(1, 128);
            float reach = 0.0f;
            for (int i = tid; i < 256; i += 128) {
                const Linear8Col c = linear8_col(p, o0 + i);
                sh.col[i] = c;
                reach = fmaxf(reach, linear8_reach(c.zp));
            }
            reach = redux_max(reach, 0xffffffffu);
            if (lane == 0) sh.reach[q] = reach;
            const bool live = row < p.N;
            const int zx = live ? __ldg(p.x_zp + row * p.x_inc) : 0;
            const float sx = live ? __ldg(p.x_step + row * p.x_inc) : 0.0f;
            named_bar_sync(1, 128);
            reach = fmaxf(fmaxf(sh.reach[0], sh.reach[1]), fmaxf(sh.reach[2], sh.reach[3]));
            bool got = mbar_wait(&sh.rx_full[acc], (it >> 1) & 1) && mbar_wait_cluster(&sh.acc_full[acc], (it >> 1) & 1);
            if (!named_bar_and(2, 128, got)) { ok = false; break; }
            tc_fence_after();
            const uint32_t rx = sh.rx[acc][q * 32 + lane];
            __syncwarp();
            if (lane == 0) mbar_arrive(&sh.rx_empty[acc]);
            const float reachK = linear8_reach(zx) * (float)p.K;
            const bool all_small = __all_sync(0xffffffffu, reachK * reach < 2.147e9f);      // see linear8_acc
            const uint32_t u = rx - (uint32_t)p.K * (uint32_t)zx;
#pragma unroll 1
            for (int c0 = 0; c0 < 256; c0 += 64) {
                if (row0 < p.N && o0 + c0 < p.O) {
#pragma unroll
                    for (int h = 0; h < 64; h += 32) {
                        uint32_t S[32];
                        tc_ld32(tmem + acc * 256 + c0 + h + ((uint32_t)(q * 32) << 16), S);
                        tc_wait_ld();
                        uint32_t packed[16];
                        if (all_small) {
#pragma unroll
                            for (int j = 0; j < 32; j += 2) {
                                const Linear8Col c = sh.col[c0 + h + j], d = sh.col[c0 + h + j + 1];
                                const float v = (float)(int)(S[j] - (uint32_t)zx * c.sum - (uint32_t)c.zp * u);
                                const float w = (float)(int)(S[j + 1] - (uint32_t)zx * d.sum - (uint32_t)d.zp * u);
                                packed[j / 2] = D::encode2(__fmaf_rn(v * sx, c.step, c.bias), __fmaf_rn(w * sx, d.step, d.bias));
                            }
                        } else {
#pragma unroll
                            for (int j = 0; j < 32; ++j) {
                                const Linear8Col c = sh.col[c0 + h + j];
                                const float v = linear8_acc(S[j], zx, rx, c.zp, c.sum, (uint32_t)p.K, reachK, reach);
                                const uint32_t y = D::encode(__fmaf_rn(v * sx, c.step, c.bias));
                                packed[j / 2] = j & 1 ? packed[j / 2] | y << 16 : y;
                            }
                        }
#pragma unroll
                        for (int j = 0; j < 4; ++j)
                            *reinterpret_cast<uint4 *>(buf + lane * kBigOutPitch + h * 2 + j * 16) =
                                make_uint4(packed[4 * j], packed[4 * j + 1], packed[4 * j + 2], packed[4 * j + 3]);
                    }
                    __syncwarp();
                    if (vec_out && o0 + c0 + 64 <= p.O) {
                        // four rows of 128 bytes per store
#pragma unroll
                        for (int i = 0; i < 8; ++i) {
                            const int r = i * 4 + (lane >> 3);
                            if (row0 + r < p.N)
                                *reinterpret_cast<uint4 *>(p.out + (row0 + r) * p.ldo + o0 + c0 + (lane & 7) * 8) =
                                    *reinterpret_cast<const uint4 *>(buf + r * kBigOutPitch + (lane & 7) * 16);
                        }
                    } else {
                        for (int r = 0; r < 32 && row0 + r < p.N; ++r)
#pragma unroll
                            for (int e = 0; e < 64; e += 32)
                                if (o0 + c0 + e + lane < p.O)
                                    p.out[(row0 + r) * p.ldo + o0 + c0 + e + lane] =
                                        *reinterpret_cast<const uint16_t *>(buf + r * kBigOutPitch + (e + lane) * 2);
                    }
                    __syncwarp();
                }
            }
            tc_fence_before();
            __syncwarp();
            if (lane == 0) cluster_mbar_arrive(cluster_map(&sh.acc_empty[acc], 0));
        }
    }
    if (!ok && p.st) atomicAdd(&p.st->wait_timeout, 1ull);
    tc_fence_before();
    __syncthreads();
    cluster_sync_all();
    if (warp == 1) tc_dealloc<2>(tmem, 512);
}

template <class D>
static aweq_status big_launch(const Linear8Args &a, cudaStream_t stream)
{
    CUtensorMap mx, mw;
    aweq_status rc = tma_bytes_map(&mx, a.X, a.N, a.K, a.ldx, 128);
    if (rc == AWEQ_OK) rc = tma_bytes_map(&mw, a.W, a.O, a.K, a.ldw, 128);
    if (rc != AWEQ_OK) return rc;
    AWEQ_CUDA_OK(cudaFuncSetAttribute(linear8_big_kernel<D>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kBigSmem));
    const int mt = (int)((a.N + 255) / 256), nt = (a.O + 255) / 256;
    const long long tiles = (long long)mt * nt;
    const unsigned pairs = (unsigned)(tiles < kSmCount / 2 ? tiles : kSmCount / 2);
    const int vec = (a.ldo % 8 == 0) && ((reinterpret_cast<uintptr_t>(a.out) & 15) == 0);
    const cudaError_t e = launch_pdl_cluster(linear8_big_kernel<D>, dim3(pairs * 2), dim3(256), kBigSmem, stream, 2, a, mx, mw, mt,
                                             nt, vec);
    note_launch();
    if (e != cudaSuccess) return cuda_failed(e);
    return AWEQ_OK;
}

aweq_status run_linear8_big(const Linear8Args &a, aweq_dtype dt, cudaStream_t stream)
{
    return dt == AWEQ_F16 ? big_launch<F16>(a, stream) : big_launch<BF16>(a, stream);
}

}  // namespace aweq
