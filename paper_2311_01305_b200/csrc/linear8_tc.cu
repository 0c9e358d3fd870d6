// aweq_linear_w8a8 on the tensor cores: tcgen05.mma kind::i8 over TMA-fed tiles.
#include <math.h>

#include "linear8.cuh"
#include "tensorcore.cuh"

namespace aweq {

constexpr int kL8Block = 128;                  // bytes of K per stage: one swizzled row

// sum of the 128 code bytes of a staged row.  A row's 16-byte pieces are permuted by the swizzle, which a
// sum does not see; the lanes start at different pieces so that they spread over the banks.
__device__ __forceinline__ uint32_t staged_row_sum(const unsigned char *row, int lane)
{
    uint32_t s[4] = {};
#pragma unroll
    for (int c = 0; c < 8; ++c) {
        const uint4 v = *reinterpret_cast<const uint4 *>(row + ((c + lane) & 7) * 16);
        s[0] = __dp4a(v.x, 0x01010101u, s[0]);
        s[1] = __dp4a(v.y, 0x01010101u, s[1]);
        s[2] = __dp4a(v.z, 0x01010101u, s[2]);
        s[3] = __dp4a(v.w, 0x01010101u, s[3]);
    }
    return (s[0] + s[1]) + (s[2] + s[3]);
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
        c.step = p.w_step[o * p.w_inc];
        c.zp = p.w_zp[o * p.w_inc];
        c.sum = (uint32_t)p.w_sum[o];
        if (p.bias) c.bias = p.bias[o];
    }
    return c;
}

// ------------------------------------------------------------------ many tokens
// Output tiles of 256 tokens x 248 channels, each by a pair of CTAs (cta_group::2): a CTA stages its 128 tokens and half of
// the weights, and holds the sums of its tokens in TMEM, twice, so that the epilogue of one tile runs under the
// products of the next.  Persistent: a pair takes every (pairs)-th tile.  Bound by the tensor pipe: 2048 x 4096 x 11008 63.5 us (2909
// TOP/s, the pipe busy 83 % of the time; calls in a row 75, at the power cap), 16384 x 5120 x 13824 711 us (3261 TOP/s); what the first
// loses is its last wave.  Warps: 0 copies, 1 issues the products (in the
// pair's even CTA), 4-11 write the output, two to a quarter of the TMEM lanes.
//
// The tokens' code sums rx come out of the same products: the last eight of the 256 rows of the weight tile are ones, laid
// down once per stage where the copies do not reach.  Summing the staged codes with other warps instead cost 14 % at 2048 x 4096
// x 11008 (the products read and the copies write 32 KB a stage each, which is all that shared memory moves in that
// time); the eight rows cost 3 %.
constexpr int kBigStages = 6, kBigThreads = 384, kBigCols = 248;
constexpr int kBigStageBytes = 2 * 128 * kL8Block;
constexpr int kBigOutPitch = 80;               // bytes of a staged output row: 32 columns and 16 bytes against bank conflicts
struct BigShared {
    uint64_t full[kBigStages], empty[kBigStages], acc_full[2], acc_empty[2];
    uint32_t tmem;
    float reach[8];
    Linear8Col col[256];
    alignas(16) unsigned char out[8][32 * kBigOutPitch];
};
constexpr size_t kBigSmem = 1024 + (size_t)kBigStages * kBigStageBytes + sizeof(BigShared);
static_assert(kBigSmem <= 227 * 1024, "shared memory of a CTA");

__device__ __forceinline__ void big_tile(long long t, int mt, int nt, int *m, int *n)
{
    // eight row blocks at a time, so that the tiles in flight share both operands in the L2
    const long long group = 8ll * nt;
    const int g = (int)(t / group), first = g * 8, height = min(8, mt - first), r = (int)(t % group);
    *m = first + r % height;
    *n = r / height;
}

template <class D>
__global__ void __launch_bounds__(kBigThreads, 1)
linear8_big_kernel(const Linear8Args p, const __grid_constant__ CUtensorMap mapX, const __grid_constant__ CUtensorMap mapW0,
                   const __grid_constant__ CUtensorMap mapW1, int mt, int nt, int vec_out)
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
            mbar_init(&sh.empty[s], 1);
        }
        for (int a = 0; a < 2; ++a) {
            mbar_init(&sh.acc_full[a], 1);
            mbar_init(&sh.acc_empty[a], 16);
        }
        mbar_init_fence();
        tma_prefetch_map(&mapX);
        tma_prefetch_map(rank ? &mapW1 : &mapW0);
    }
    if (rank == 1) {                               // rows 120-127 of this CTA's half of the weight tile: ones
        for (int i = threadIdx.x; i < kBigStages * 64; i += kBigThreads)
            *reinterpret_cast<uint4 *>(stages + (i >> 6) * kBigStageBytes + (128 + 120) * kL8Block + (i & 63) * 16) =
                make_uint4(0x01010101u, 0x01010101u, 0x01010101u, 0x01010101u);
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
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
            const CUtensorMap *const mapW = rank ? &mapW1 : &mapW0;
            int s = 0;
            uint32_t ph = 0;
            for (long long t = blockIdx.x / 2; ok && t < tiles; t += step) {
                int m, n;
                big_tile(t, mt, nt, &m, &n);
                const int row = m * 256 + (int)rank * 128, col = n * kBigCols + (int)rank * 128;
                for (int kb = 0; kb < nkb; ++kb) {
                    if (!mbar_wait_cluster(&sh.empty[s], ph ^ 1)) { ok = false; break; }
                    const uint32_t bar = cluster_map(&sh.full[s], 0), dst = smem_u32(stages + s * kBigStageBytes);
                    if (rank == 0) mbar_arrive_expect_tx(&sh.full[s], 2 * kBigStageBytes - 8 * kL8Block);
                    tma_load2<2>(dst, &mapX, kb * kL8Block, row, bar);
                    tma_load2<2>(dst + 128 * kL8Block, mapW, kb * kL8Block, col, bar);
                    if (++s == kBigStages) { s = 0; ph ^= 1; }
                }
            }
            if (!ok && rank == 0)              // gave up: let what is under way land (bounded) before the memory goes
                for (int i = 0; i < kBigStages; ++i) mbar_wait(&sh.full[i], ph ^ (i >= s ? 1u : 0u));
        }
    } else if (warp == 1) {
        if (rank == 0) {
            const bool lead = tc_elect();
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
                    const uint32_t da = tc_desc(a), db = tc_desc(a + 128 * kL8Block);
#pragma unroll
                    for (int k = 0; k < 4; ++k)
                        tc_mma_u8<2>(tmem + acc * 256, da + 2 * k, db + 2 * k, idesc, (kb | k) != 0, lead);
                    tc_commit<2>(&sh.empty[s], lead);
                    if (++s == kBigStages) { s = 0; ph ^= 1; }
                }
                if (ok) tc_commit<2>(&sh.acc_full[acc], lead);
            }
        }
    } else if (warp >= 4) {
        const int q = warp & 3, half = (warp - 4) >> 2, tid = threadIdx.x - 128;
        unsigned char *buf = sh.out[warp - 4];
        int it = 0;
        for (long long t = blockIdx.x / 2; t < tiles; t += step, ++it) {
            const int acc = it & 1;
            int m, n;
            big_tile(t, mt, nt, &m, &n);
            const long long row0 = (long long)m * 256 + rank * 128 + q * 32, row = row0 + lane, o0 = (long long)n * kBigCols;
            // the channels' pairs, and the largest reach of their zero-points
            named_bar_sync(1, 256);
            const Linear8Col mine = linear8_col(p, tid < kBigCols ? o0 + tid : p.O);
            sh.col[tid] = mine;
            float reach = redux_max(linear8_reach(mine.zp), 0xffffffffu);
            if (lane == 0) sh.reach[warp - 4] = reach;
            const bool live = row < p.N;
            const int zx = live ? p.x_zp[row * p.x_inc] : 0;
            const float sx = live ? p.x_step[row * p.x_inc] : 0.0f;
            named_bar_sync(1, 256);
#pragma unroll
            for (int i = 0; i < 8; ++i) reach = fmaxf(reach, sh.reach[i]);
            const bool got = mbar_wait_cluster(&sh.acc_full[acc], (it >> 1) & 1);
            if (!named_bar_and(2, 256, got)) { ok = false; break; }
            tc_fence_after();
            const uint32_t at = tmem + acc * 256 + ((uint32_t)(q * 32) << 16);
            if (row0 < p.N) {
                const uint32_t rx = tc_ld1(at + kBigCols);
                const float reachK = linear8_reach(zx) * (float)p.K;
                const bool all_small = __all_sync(0xffffffffu, reachK * reach < 2.147e9f);      // see linear8_acc
                const uint32_t u = rx - (uint32_t)p.K * (uint32_t)zx;
                const int c1 = half ? kBigCols : 128;
#pragma unroll 1
                for (int c0 = half * 128; c0 < c1 && o0 + c0 < p.O; c0 += 32) {
                    uint32_t S[32], packed[16];
                    tc_ld32(at + c0, S);
                    tc_wait_ld();
                    if (all_small) {
#pragma unroll
                        for (int j = 0; j < 32; j += 2) {
                            const Linear8Col c = sh.col[c0 + j], d = sh.col[c0 + j + 1];
                            const float v = (float)(int)(S[j] - (uint32_t)zx * c.sum - (uint32_t)c.zp * u);
                            const float w = (float)(int)(S[j + 1] - (uint32_t)zx * d.sum - (uint32_t)d.zp * u);
                            packed[j / 2] = D::encode2(__fmaf_rn(v * sx, c.step, c.bias), __fmaf_rn(w * sx, d.step, d.bias));
                        }
                    } else {
#pragma unroll
                        for (int j = 0; j < 32; ++j) {
                            const Linear8Col c = sh.col[c0 + j];
                            const float v = linear8_acc(S[j], zx, rx, c.zp, c.sum, (uint32_t)p.K, reachK, reach);
                            const uint32_t y = D::encode(__fmaf_rn(v * sx, c.step, c.bias));
                            packed[j / 2] = j & 1 ? packed[j / 2] | y << 16 : y;
                        }
                    }
#pragma unroll
                    for (int j = 0; j < 4; ++j)
                        *reinterpret_cast<uint4 *>(buf + lane * kBigOutPitch + j * 16) =
                            make_uint4(packed[4 * j], packed[4 * j + 1], packed[4 * j + 2], packed[4 * j + 3]);
                    __syncwarp();
                    const int cols = (int)min((long long)min(32, c1 - c0), p.O - (o0 + c0));
                    if (vec_out && cols % 8 == 0) {
                        // eight rows of 64 bytes per store
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            const int r = i * 8 + (lane >> 2), c = (lane & 3) * 8;
                            if (row0 + r < p.N && c < cols)
                                *reinterpret_cast<uint4 *>(p.out + (row0 + r) * p.ldo + o0 + c0 + c) =
                                    *reinterpret_cast<const uint4 *>(buf + r * kBigOutPitch + c * 2);
                        }
                    } else {
                        for (int r = 0; r < 32 && row0 + r < p.N; ++r)
                            if (lane < cols) p.out[(row0 + r) * p.ldo + o0 + c0 + lane] = *reinterpret_cast<const uint16_t *>(buf + r * kBigOutPitch + lane * 2);
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
    CUtensorMap mx, w0, w1;
    aweq_status rc = tma_bytes_map(&mx, a.X, a.N, a.K, a.ldx, 128);
    if (rc == AWEQ_OK) rc = tma_bytes_map(&w0, a.W, a.O, a.K, a.ldw, 128);
    if (rc == AWEQ_OK) rc = tma_bytes_map(&w1, a.W, a.O, a.K, a.ldw, 120);
    if (rc != AWEQ_OK) return rc;
    static std::atomic<unsigned long long> allowed{0};
    AWEQ_CUDA_OK(allow_smem(linear8_big_kernel<D>, kBigSmem, allowed));
    const int mt = (int)((a.N + 255) / 256), nt = (a.O + kBigCols - 1) / kBigCols;
    const long long tiles = (long long)mt * nt;
    const unsigned pairs = (unsigned)(tiles < kSmCount / 2 ? tiles : kSmCount / 2);
    const int vec = (a.ldo % 8 == 0) && ((reinterpret_cast<uintptr_t>(a.out) & 15) == 0);
    const cudaError_t e = launch_pdl_cluster(linear8_big_kernel<D>, dim3(pairs * 2), dim3(kBigThreads), kBigSmem, stream, 2, a, mx, w0, w1,
                                             mt, nt, vec);
    note_launch();
    if (e != cudaSuccess) return cuda_failed(e);
    return AWEQ_OK;
}

static aweq_status run_linear8_big(const Linear8Args &a, aweq_dtype dt, cudaStream_t stream)
{
    return dt == AWEQ_F16 ? big_launch<F16>(a, stream) : big_launch<BF16>(a, stream);
}

// ------------------------------------------------------------------ a moderate number of tokens
// The layer is bound by the weights here: what counts is that every SM has a deep queue of copies under
// way and that they all end together.  A CTA per SM takes up to 256 tokens x bn channels, with bn chosen so that
// the tiles fill one wave; where few channels leave SMs idle, K is cut over the CTAs of a cluster, whose integer
// sums are added through distributed shared memory (exact in any order), each CTA finishing its share of the
// rows.  A stage holds the tokens there are (rounded up to 8), not 128, so that few tokens leave the ring to the
// weights; the product reads 128 rows all the same, those past the box belong to the weights behind them and
// give sums that nobody reads.  Warps: 0 copies, 1 issues the products, 2-7 add up the tokens' codes.  The sums go
// through shared memory (the stages) once so that the output is written along the channels.  Measured on the device: 16 x 4096 x 12288 12.5 us;
// 16 x 9216 x 36864 56 us, 6.1 TB/s; 64 x 4096 x 4096 10.9 us (its start and its end).
constexpr int kSplitRing = 200 * 1024, kSplitMaxStages = 16;
struct SplitPlan {
    int bn, slices;              // channels of a tile, slices of K
    int box, mb;                 // token rows of a stage, 128-row blocks they make
    int stages, kb_stage;        // ring, 128-byte blocks of K per stage
    int rx_groups, rx_sets;      // 32-row groups of a stage; warps that share a group's stages
};
struct alignas(16) Linear8Row {
    float step, reachK;
    int zp;
    uint32_t rx;
};
struct SplitShared {
    uint64_t full[kSplitMaxStages], empty[kSplitMaxStages], acc_full;
    uint32_t tmem, rx[256];
    Linear8Row row[256];
    Linear8Col col[256];
};
constexpr size_t kSplitSmem = 1024 + kSplitRing + sizeof(SplitShared);
static_assert(kSplitSmem <= 227 * 1024, "shared memory of a CTA");

template <class D>
__global__ void __launch_bounds__(256, 1)
linear8_split_kernel(const Linear8Args p, const __grid_constant__ CUtensorMap mapX, const __grid_constant__ CUtensorMap mapW,
                     const SplitPlan plan, int vec_out)
{
    extern __shared__ unsigned char raw[];
    unsigned char *stages = reinterpret_cast<unsigned char *>((reinterpret_cast<uintptr_t>(raw) + 1023) & ~(uintptr_t)1023);
    SplitShared &sh = *reinterpret_cast<SplitShared *>(stages + kSplitRing);
    uint32_t *part = reinterpret_cast<uint32_t *>(stages);
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int bn = plan.bn, pitch = bn + 4, x_bytes = plan.box * kL8Block, kb_bytes = x_bytes + bn * kL8Block;
    const int slices = plan.slices, slice = blockIdx.x;
    const int nkb = (p.K + kL8Block - 1) / kL8Block;
    const int kb0 = (int)((long long)nkb * slice / slices), kb1 = (int)((long long)nkb * (slice + 1) / slices);
    const long long row0 = (long long)blockIdx.z * 128 * plan.mb;
    const int rows = (int)min(128ll * plan.mb, p.N - row0);
    const int o0 = blockIdx.y * bn;
    uint32_t cols = 32;
    while ((int)cols < bn * plan.mb) cols *= 2;
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    if (threadIdx.x == 0) {
        for (int s = 0; s < plan.stages; ++s) {
            mbar_init(&sh.full[s], 1);
            mbar_init(&sh.empty[s], 1 + min(plan.rx_groups, 6));
        }
        mbar_init(&sh.acc_full, 1);
        mbar_init_fence();
        tma_prefetch_map(&mapX);
        tma_prefetch_map(&mapW);
    }
    sh.rx[threadIdx.x] = 0;
    if (warp == 1) tc_alloc<1>(&sh.tmem, cols);
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
            for (int kb = kb0; kb < kb1; kb += plan.kb_stage) {
                if (!mbar_wait(&sh.empty[s], ph ^ 1)) { ok = false; break; }
                const int n = min(plan.kb_stage, kb1 - kb);
                uint32_t dst = smem_u32(stages + s * plan.kb_stage * kb_bytes);
                const uint32_t bar = smem_u32(&sh.full[s]);
                mbar_arrive_expect_tx(&sh.full[s], (uint32_t)(n * kb_bytes));
                for (int i = 0; i < n; ++i, dst += kb_bytes) {
                    tma_load2<1>(dst + x_bytes, &mapW, (kb + i) * kL8Block, o0, bar);
                    tma_load2<1>(dst, &mapX, (kb + i) * kL8Block, (int)row0, bar);
                }
                if (++s == plan.stages) { s = 0; ph ^= 1; }
            }
            if (!ok)                           // gave up: let what is under way land (bounded) before the memory goes
                for (int i = 0; i < plan.stages; ++i) mbar_wait(&sh.full[i], ph ^ (i >= s ? 1u : 0u));
        }
    } else if (warp == 1) {
        const bool lead = tc_elect();
        int s = 0;
        uint32_t ph = 0;
        const uint32_t idesc = tc_idesc_u8(128, bn);
        for (int kb = kb0; kb < kb1; kb += plan.kb_stage) {
            if (!mbar_wait(&sh.full[s], ph)) { ok = false; break; }
            tc_fence_after();
            const int n = min(plan.kb_stage, kb1 - kb);
            uint32_t a = smem_u32(stages + s * plan.kb_stage * kb_bytes);
            for (int i = 0; i < n; ++i, a += kb_bytes) {
                const uint32_t da = tc_desc(a), db = tc_desc(a + x_bytes);
                for (int b = 0; b < plan.mb; ++b)
#pragma unroll
                    for (int k = 0; k < 4; ++k)
                        tc_mma_u8<1>(tmem + b * bn, da + b * (128 * kL8Block / 16) + 2 * k, db + 2 * k, idesc, kb + i > kb0 || k > 0, lead);
            }
            tc_commit<1>(&sh.empty[s], lead);
            if (++s == plan.stages) { s = 0; ph ^= 1; }
        }
        if (ok) {
            tc_commit<1>(&sh.acc_full, lead);
            ok = mbar_wait(&sh.acc_full, 0);
        }
    } else {
        // the pairs of channels and tokens, while the first copies are under way
        for (int i = threadIdx.x - 64; i < bn; i += 192) sh.col[i] = linear8_col(p, o0 + i);
        for (int i = threadIdx.x - 64; i < rows; i += 192) {
            const int z = p.x_zp[(row0 + i) * p.x_inc];
            sh.row[i] = {p.x_step[(row0 + i) * p.x_inc], linear8_reach(z) * (float)p.K, z, 0u};
        }
        const int groups = min(plan.rx_groups, 6), group = (warp - 2) % groups, set = (warp - 2) / groups;
        if (set < plan.rx_sets) {
            // rows group * 32 + lane and, from 193 rows on, 192 further (boxes hold at most 256), in every rx_sets-th
            // stage of the ring: a warp sees every phase of the barriers that it waits on
            const int ra = group * 32 + lane, rb = ra + 192;
            const bool two = group * 32 + 192 < plan.box;
            int s = 0;
            uint32_t ph = 0, a = 0, b = 0;
            for (int kb = kb0; kb < kb1; kb += plan.kb_stage) {
                if (s % plan.rx_sets == set) {
                    ok = mbar_wait(&sh.full[s], ph);
                    if (!__all_sync(0xffffffffu, ok)) { ok = false; break; }
                    const unsigned char *x = stages + s * plan.kb_stage * kb_bytes;
                    const int n = min(plan.kb_stage, kb1 - kb);
                    for (int i = 0; i < n; ++i, x += kb_bytes) {
                        a += staged_row_sum(x + ra * kL8Block, lane);
                        if (two) b += staged_row_sum(x + rb * kL8Block, lane);
                    }
                    __syncwarp();
                    if (lane == 0) mbar_arrive(&sh.empty[s]);
                }
                if (++s == plan.stages) { s = 0; ph ^= 1; }
            }
            atomicAdd(&sh.rx[ra], a);
            if (two) atomicAdd(&sh.rx[rb], b);
        }
    }
    // every product, copy and row sum of this CTA is done (or has been given up)
    if (!ok && p.st) atomicAdd(&p.st->wait_timeout, 1ull);
    __syncthreads();
    tc_fence_after();
    {
        // warps 0-3 and 4-7 take the blocks' four TMEM quarters in turn (a warp reads quarter warp % 4)
        const int q = warp & 3;
        const int b0 = plan.mb == 2 ? warp >> 2 : 0, c0 = plan.mb == 2 ? 0 : (warp >> 2) * 32, dc = plan.mb == 2 ? 32 : 64;
        const int r = b0 * 128 + q * 32;
        if (r < rows)
            for (int c = c0; c < bn; c += dc) {
                uint32_t S[32];
                tc_ld32(tmem + b0 * bn + c + ((uint32_t)(q * 32) << 16), S);
                tc_wait_ld();
                if (r + lane < rows)
#pragma unroll
                    for (int j = 0; j < 32; j += 4)
                        *reinterpret_cast<uint4 *>(part + (r + lane) * pitch + c + j) = make_uint4(S[j], S[j + 1], S[j + 2], S[j + 3]);
            }
    }
    tc_fence_before();
    if (slices > 1) cluster_sync_all();
    else __syncthreads();
    if (warp == 1) {
        __syncwarp();
        tc_fence_after();
        tc_dealloc<1>(tmem, cols);
    }
    // rows slice, slice + slices, ... are this CTA's
    for (int r = threadIdx.x; r < rows; r += 256)
        if (r % slices == slice) {
            uint32_t rx = sh.rx[r];
            for (int k = 1; k < slices; ++k) {
                uint32_t x;
                asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(x) : "r"(cluster_map(sh.rx + r, (slice + k) % slices)) : "memory");
                rx += x;
            }
            sh.row[r].rx = rx;
        }
    __syncthreads();
    // a warp per row, a lane per pair of channels, four rows in flight
    constexpr int U = 4;
    for (int rb = slice + slices * warp; rb < rows; rb += slices * 8 * U)
        for (int c = lane * 2; c < bn; c += 64) {
            uint2 S[U];
#pragma unroll
            for (int u = 0; u < U; ++u)
                S[u] = *reinterpret_cast<const uint2 *>(part + min(rb + u * slices * 8, rows - 1) * pitch + c);
            for (int k = 1; k < slices; ++k) {
                const uint32_t peer = cluster_map(part + c, (slice + k) % slices);
                uint2 v[U];
#pragma unroll
                for (int u = 0; u < U; ++u)
                    asm volatile("ld.shared::cluster.v2.u32 {%0,%1}, [%2];" : "=r"(v[u].x), "=r"(v[u].y)
                                 : "r"(peer + min(rb + u * slices * 8, rows - 1) * pitch * 4) : "memory");
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    S[u].x += v[u].x;
                    S[u].y += v[u].y;
                }
            }
            const Linear8Col a = sh.col[c], b = sh.col[c + 1];
            const float reach_a = linear8_reach(a.zp), reach_b = linear8_reach(b.zp);
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int r = rb + u * slices * 8;
                if (r >= rows) break;
                const Linear8Row x = sh.row[r];
                const float va = linear8_acc(S[u].x, x.zp, x.rx, a.zp, a.sum, (uint32_t)p.K, x.reachK, reach_a);
                const float vb = linear8_acc(S[u].y, x.zp, x.rx, b.zp, b.sum, (uint32_t)p.K, x.reachK, reach_b);
                const float ya = __fmaf_rn(va * x.step, a.step, a.bias), yb = __fmaf_rn(vb * x.step, b.step, b.bias);
                uint16_t *dst = p.out + (row0 + r) * p.ldo + o0 + c;
                if (vec_out && o0 + c + 2 <= p.O)
                    *reinterpret_cast<uint32_t *>(dst) = D::encode2(ya, yb);
                else {
                    if (o0 + c < p.O) dst[0] = D::encode(ya);
                    if (o0 + c + 1 < p.O) dst[1] = D::encode(yb);
                }
            }
        }
    if (slices > 1) cluster_sync_all();        // nobody leaves while its sums may still be read
}

template <class D>
static aweq_status split_launch(const Linear8Args &a, SplitPlan plan, cudaStream_t stream)
{
    CUtensorMap mx, mw;
    aweq_status rc = tma_bytes_map(&mx, a.X, a.N, a.K, a.ldx, plan.box);
    if (rc == AWEQ_OK) rc = tma_bytes_map(&mw, a.W, a.O, a.K, a.ldw, plan.bn);
    if (rc != AWEQ_OK) return rc;
    static std::atomic<unsigned long long> allowed{0};
    AWEQ_CUDA_OK(allow_smem(linear8_split_kernel<D>, kSplitSmem, allowed));
    const dim3 grid((unsigned)plan.slices, (unsigned)((a.O + plan.bn - 1) / plan.bn), (unsigned)((a.N + 128 * plan.mb - 1) / (128 * plan.mb)));
    const int vec = (a.ldo % 2 == 0) && ((reinterpret_cast<uintptr_t>(a.out) & 3) == 0);
    const cudaError_t e = launch_pdl_cluster(linear8_split_kernel<D>, grid, dim3(256), kSplitSmem, stream, (unsigned)plan.slices, a, mx,
                                             mw, plan, vec);
    note_launch();
    if (e != cudaSuccess) return cuda_failed(e);
    return AWEQ_OK;
}

// Which kernel, and how it cuts the layer.
//
// The plain-load kernel (linear8.cu) reads the weights once for up to 32 tokens and the tokens once for every 16 channels: it wins
// while that is little (1 x 4096 x 4096: 6.8 us against 7.7; 64 x 768 x 768: 3.6 against 5.5; 16 x 4096 x 12288: 19.1 against 12.7).
// For the other two the estimate below is within about 10 % of 70 measured (shape, cut) pairs between 16 x 4096 x 4096
// and 256 x 4096 x 4096, in microseconds: a start, then per 128-byte block of K the slowest of an issue limit, what an SM
// can take in and what the memory gives.  A K slice costs an exchange; clusters of three and four do not fill the device.
struct Linear8Choice {
    int kernel;                  // 0: plain loads, 1: K slices on single CTAs, 2: pairs of CTAs
    int bn, slices;
};
static Linear8Choice linear8_choose(long long N, int K, int O)
{
    if (N <= 64 && (double)K * O * (double)(N > 16 ? N : 16) <= 2.7e8) return {0, 0, 0};
    const int nkb = (K + kL8Block - 1) / kL8Block;
    const double tiles = (double)((N + 255) / 256) * ((O + kBigCols - 1) / kBigCols), waves = ceil(tiles / (kSmCount / 2));
    Linear8Choice best = {2, 0, 0};
    double cost = 6.0 + waves * nkb * (0.3 + 0.1 * (tiles < 60 ? tiles / 60 : 1.0));
    static const int bns[5] = {32, 64, 96, 128, 256}, most[5] = {0, kSmCount, kSmCount, 120, 128};
    if (N <= 256)
        for (int bn : bns) {
            if ((O + bn - 1) / bn > 65535) continue;             // channels lie on the grid's second dimension
            for (int slices = 1; slices <= 4 && slices <= nkb; ++slices) {
                const int mb = N > 128 && bn <= 128 ? 2 : 1;
                const double rows = N < 128 * mb ? (double)N : 128.0 * mb, box = rows + 7;
                const double ctas = (double)((O + bn - 1) / bn) * (double)((N + 128 * mb - 1) / (128 * mb)) * slices;
                if (slices > 1 && ctas > most[slices]) continue;
                const double live = ctas < kSmCount ? ctas : kSmCount;
                double t = 0.16;
                t = fmax(t, (bn + box) * 128 / 75e3);
                t = fmax(t, bn * 128 * live / 6.6e6);
                if (bn >= 128) t = fmax(t, 0.13 * mb * bn / 128);
                const double c = 4.6 + ceil(ctas / kSmCount) * ((nkb + slices - 1) / slices * t + 0.00012 * rows * bn / slices) +
                                 (slices > 1 ? 0.9 + 0.009 * rows : 0.0);
                if (c < cost) {
                    cost = c;
                    best = {1, bn, slices};
                }
            }
        }
    return best;
}

static aweq_status run_linear8_split(const Linear8Args &a, aweq_dtype dt, int bn, int slices, cudaStream_t stream)
{
    SplitPlan s;
    s.mb = a.N > 128 && bn <= 128 ? 2 : 1;
    const long long rows = a.N < 128 * s.mb ? a.N : 128 * s.mb;
    s.bn = bn;
    s.slices = slices;
    s.box = (int)((rows + 7) / 8 * 8);
    const int kb_bytes = (s.box + bn) * kL8Block, span = s.mb * 128 * kL8Block;
    s.kb_stage = kb_bytes <= 20 * 1024 ? 2 : 1;
    // the product's 128 rows per block stay inside the ring from the last block of K on too
    const int blocks = (kSplitRing - (span > kb_bytes ? span : kb_bytes)) / kb_bytes + 1;
    s.stages = blocks / s.kb_stage;
    if (s.stages > kSplitMaxStages) s.stages = kSplitMaxStages;
    s.rx_groups = (s.box + 31) / 32;
    s.rx_sets = s.rx_groups <= 3 ? 6 / s.rx_groups : 1;
    return dt == AWEQ_F16 ? split_launch<F16>(a, s, stream) : split_launch<BF16>(a, s, stream);
}

aweq_status run_linear8(const Linear8Args &a, aweq_dtype dt, cudaStream_t stream)
{
    const Linear8Choice c = linear8_choose(a.N, a.K, a.O);
    if (c.kernel == 0) return run_linear8_stream(a, dt, stream);
    if (c.kernel == 1) return run_linear8_split(a, dt, c.bn, c.slices, stream);
    return run_linear8_big(a, dt, stream);
}

}  // namespace aweq
