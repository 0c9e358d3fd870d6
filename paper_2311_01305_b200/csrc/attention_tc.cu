// The prefix part of aweq_prefix_attention on the tensor cores (tcgen05), for many rows and for page sizes whose rows keep
// the swizzle's phase.
//
// An item is up to 128 rows (TMEM lanes) against the prefix, 128 keys (or the whole pages that fit) to a unit:
//   S = Q K^T   A = Q in TMEM, B = the staged keys            -> S in TMEM (two buffers)
//   P = 2^((S - m) scale)  by two threads per row, 16-bit, in TMEM over the S it came from
//   O += P V    A = P in TMEM, B = the staged values (N contiguous)  -> O in TMEM
// Each row's reference maximum m moves only when a new maximum exceeds it by more than 8 (a factor of 256, for which
// the 16-bit P and the binary32 sums have room), so O is hardly ever rescaled: only then do the softmax threads
// wait for the product under way, scale O and go on.
// What bounds it: one unit's chain of load, maximum, meeting, exponentials and store, 2800 cycles, in which neither the exponentials'
// pipe (1060 cycles) nor the tensor pipe (37 %) is full (384 rows x 32779 keys x 8 heads of 128: 73 us by itself, 0.71 PFLOP/s).
// Warps: 0 and 2 look up pages and issue the copies of K and V, 1 issues the products (S of a unit before O of the one
// before it), 4-11 softmax (two threads to a row, half of the keys each), 12-15 bring the next item's rows of Q and take
// the finished item's O to its record.
#include "attention.cuh"
#include "tensorcore.cuh"

namespace aweq {

constexpr int kTcThreads = 512, kTcStageBytes = 192 * 1024, kTcMaxStages = 6;
constexpr uint32_t kTcO = 256, kTcQ = 384;      // TMEM columns: S at 0 and 128, O, two of Q (64 columns each)
constexpr float kTcSlack = 8.0f;

// A unit: the tile'th tile of the prefix for row tile rt of key head kh.
struct alignas(16) TcUnit {
    int kh, rt, tile, keys;
    int leave, stop, item, fresh;        // last / first of its item in this CTA; last of all; number of the item here
};
// Rows of an item, and the first row of its record.
struct TcItem {
    int nrows, row0;
    long long rec;
};
__device__ __forceinline__ TcItem tc_item(const AttentionArgs &a, const AttentionPlan &p, int kh, int rt, int cta)
{
    const int rows = (int)a.n_seq * a.n_q * (a.n_heads / a.n_kv) - rt * 128;
    return {min(rows, 128), rt * 128, (long long)(kh * p.pre_rt + rt + cta) * p.pre_rec};
}

struct TcShared {
    uint64_t full[kTcMaxStages], empty[kTcMaxStages], s_full[2], p_ready[2], pv_done[2], q_ready[2], item_done[4], o_full, o_free;
    TcUnit unit[kTcMaxStages];
    uint32_t tmem;
    volatile int gave_up[4];             // by TMEM quarter: a softmax warp has
    float top[2][2][128], sum[128];      // the halves' maxima (by unit parity), one half's sum
};
constexpr size_t kTcSmem = 1024 + kTcStageBytes + sizeof(TcShared);

template <class D>
__global__ void __launch_bounds__(kTcThreads, 1)
attention_tc_kernel(const AttentionArgs a, const AttentionPlan p, const __grid_constant__ CUtensorMap mapK,
                    const __grid_constant__ CUtensorMap mapV, unsigned char *ws)
{
    extern __shared__ unsigned char raw[];
    unsigned char *const stages = reinterpret_cast<unsigned char *>((reinterpret_cast<uintptr_t>(raw) + 1023) & ~(uintptr_t)1023);
    TcShared &sh = *reinterpret_cast<TcShared *>(stages + kTcStageBytes);
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, cta = blockIdx.x, hd = a.head_dim;
    const int halves = hd > 64 ? 2 : 1, nstages = kTcStageBytes / (2 * halves * 16384), v_at = halves * 16384, stage_bytes = 2 * v_at;
    if (tid == 0) {
        for (int i = 0; i < nstages; ++i) {
            mbar_init(&sh.full[i], 2);
            mbar_init(&sh.empty[i], 1);
        }
        for (int i = 0; i < 2; ++i) {
            mbar_init(&sh.s_full[i], 1);
            mbar_init(&sh.p_ready[i], 8);
            mbar_init(&sh.pv_done[i], 1);
            mbar_init(&sh.q_ready[i], 4);
        }
        mbar_init(&sh.o_full, 1);
        mbar_init(&sh.o_free, 4);
        for (int i = 0; i < 4; ++i) {
            mbar_init(&sh.item_done[i], 8);
            sh.gave_up[i] = 0;
        }
        mbar_init_fence();
        tma_prefetch_map(&mapK);
        tma_prefetch_map(&mapV);
    }
    if (warp == 1) tc_alloc<1>(&sh.tmem, 512);
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = sh.tmem;
    // the kernel of the own keys may start as soon as what came before this one is done: it does not wait for this one
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    const AttentionDeal deal(p.pre_units, p.tc_ctas);
    const long long u0 = deal.first(cta);
    const int units = (int)(deal.first(cta + 1) - u0), item0 = (int)div_units(u0, (int)p.pre_tiles), tile0 = (int)(u0 - item0 * p.pre_tiles);
    // the CTA's items are item0, item0 + 1, ...: key head item / pre_rt, row tile item % pre_rt

    bool ok = true;
    if (warp < 4) {
        if (warp == 0 || warp == 2) {
            // ---------------------------------------------------------- copies: warp 0 of K, warp 2 of V
            const bool lead = warp == 0;
            const CUtensorMap *const map = lead ? &mapK : &mapV;
            const int boxes = p.pre_unit / p.box;
            auto has = [&](int tile) { return lane < boxes && (long long)tile * p.pre_unit + lane * p.box < a.prefix_len; };
            auto look_up = [&](int tile) {                                  // entry of the lane's box (not looked at here: the load flies)
                return has(tile) ? __ldg(a.prefix_pages + (unsigned)(tile * p.pre_unit + lane * p.box) / (unsigned)a.page_size) : 0;
            };
            int tile = tile0, kh = item0 / p.pre_rt, rt = item0 % p.pre_rt, page = look_up(tile), s = 0, items = 0;
            uint32_t ph = 0;
            bool fresh = true;
            for (int left = units; left > 0; --left) {
                TcUnit u;
                u.kh = kh;
                u.rt = rt;
                u.tile = tile;
                u.keys = (int)min((long long)p.pre_unit, a.prefix_len - (long long)tile * p.pre_unit);
                u.stop = left == 1;
                u.leave = tile + 1 == p.pre_tiles || u.stop;
                u.item = items;
                u.fresh = fresh;
                const bool there = has(u.tile), bad = bad_page(a, page);
                const int pid = bad ? 0 : page;
                if (++tile == p.pre_tiles) {
                    tile = 0;
                    if (++rt == p.pre_rt) { rt = 0; ++kh; }
                }
                if (left > 1) page = look_up(tile);                         // the next unit's, while this stage empties
                ok = mbar_wait(&sh.empty[s], ph ^ 1);
                if (!__all_sync(0xffffffffu, ok)) { ok = false; break; }
                const int n = __popc(__ballot_sync(0xffffffffu, there));
                if (lane == 0) {
                    if (lead) sh.unit[s] = u;
                    mbar_arrive_expect_tx(&sh.full[s], (uint32_t)(n * p.box * 128 * halves));
                }
                __syncwarp();
                if (there) {
                    const uint32_t dst = smem_u32(stages + s * stage_bytes + (lead ? 0 : v_at)) + lane * p.box * 128, bar = smem_u32(&sh.full[s]);
                    const int row = (unsigned)(u.tile * p.pre_unit + lane * p.box) % (unsigned)a.page_size;
                    if (lead && bad) count_bad_page(a, u.kh, u.rt, row);
                    for (int h = 0; h < halves; ++h) tma_load4(dst + h * 16384, map, h * 64, u.kh, row, pid, bar);
                }
                fresh = u.leave;
                items += u.leave;
                if (++s == nstages) { s = 0; ph ^= 1; }
            }
            if (!ok)                                                        // gave up: let what is under way land (bounded)
                for (int i = 0; i < nstages; ++i) mbar_wait(&sh.full[i], ph ^ (i >= s ? 1u : 0u));
        } else if (warp == 1) {
            // ---------------------------------------------------------- products
            const bool lead = tc_elect();
            const uint32_t idesc_s = tc_idesc_f16(D::kBf16, 128, 128, false), idesc_o = tc_idesc_f16(D::kBf16, 128, (hd + 15) / 16 * 16, true);
            const int ksteps = (hd + 15) / 16;
            int s = 0, u = 0;
            uint32_t ph = 0;
            TcUnit it, next;
            auto scores = [&](int stage, int uu, const TcUnit &x) {  // S of a unit whose stage has landed
                if (x.fresh && !mbar_wait(&sh.q_ready[x.item & 1], (x.item >> 1) & 1)) return false;
                tc_fence_after();
                const uint32_t k = tc_desc(smem_u32(stages) + stage * stage_bytes), q = tmem + kTcQ + (x.item & 1) * 64;
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    if (i < ksteps) tc_mma_f16_ta(tmem + (uu & 1) * 128, q + i * 8, k + (i >> 2) * 1024 + 2 * (i & 3), idesc_s, i > 0, lead);
                tc_commit<1>(&sh.s_full[uu & 1], lead);
                return true;
            };
            ok = mbar_wait(&sh.full[0], 0);
            if (ok) {
                it = sh.unit[0];
                ok = scores(0, 0, it);
            }
            while (ok) {
                const int s1 = s + 1 == nstages ? 0 : s + 1;
                const uint32_t ph1 = s1 ? ph : ph ^ 1;
                if (!it.stop) {
                    if (!(ok = mbar_wait(&sh.full[s1], ph1))) break;
                    next = sh.unit[s1];
                    if (!(ok = scores(s1, u + 1, next))) break;
                }
                if (!(ok = mbar_wait(&sh.p_ready[u & 1], (u >> 1) & 1))) break;
                if (it.fresh && it.item > 0 && !(ok = mbar_wait(&sh.o_free, (it.item - 1) & 1))) break;
                tc_fence_after();
                const uint32_t v = tc_desc_mn(smem_u32(stages) + s * stage_bytes + v_at, 16384);
                const int steps = (it.keys + 15) / 16;
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    if (i < steps) tc_mma_f16_ta(tmem + kTcO, tmem + (u & 1) * 128 + i * 8, v + i * 128, idesc_o, !it.fresh || i > 0, lead);
                tc_commit<1>(&sh.empty[s], lead);
                tc_commit<1>(&sh.pv_done[u & 1], lead);
                if (it.leave) tc_commit<1>(&sh.o_full, lead);
                if (it.stop) break;
                it = next;
                s = s1;
                ph = ph1;
                ++u;
            }
        }
    } else if (warp < 12) {
        // -------------------------------------------------------------- softmax: two threads per row
        const int q4 = warp & 3, half = (warp - 4) >> 2, r = q4 * 32 + lane, st = tid - 128;
        const uint32_t lanes = (uint32_t)(q4 * 32) << 16;
        // a negative scale turned q's signs; a zero one must leave -inf where a key is not seen
        const float scale = (a.scale == 0.0f ? 1.17549435e-38f : fabsf(a.scale)) * 1.4426950408889634f;
        // The row's reference is a score before scaling: the difference to it is taken first and scaled then, which is as good as the
        // scores are, however large.  (One step, the rounded scaled maximum taken off an unrounded product, gives infinity or zero
        // from 2^28 on.  Two steps on pairs of scores cost 384 rows x 32779 keys 1 us, on single ones 2.5.)
        constexpr float kShift = D::kBf16 ? 0.0f : kProbabilityShift;
        float m = -CUDART_INF_F, l = 0.0f;
        int s = 0, u = 0, nrows = 0;
        uint32_t ph = 0;
        long long rec = 0;
        // The two warps that share 32 rows wait for one another; one that gives up says so and arrives for the other.
        auto meet = [&] {
            named_bar_sync(2 + q4, 64);
            return !sh.gave_up[q4];
        };
        for (;; ++u) {
            ok = mbar_wait(&sh.full[s], ph);
            if (!__all_sync(0xffffffffu, ok)) { ok = false; break; }
            const TcUnit it = sh.unit[s];
            if (it.fresh) {
                const TcItem x = tc_item(a, p, it.kh, it.rt, cta);
                nrows = x.nrows;
                rec = x.rec;
                l = 0.0f;
            }
            const bool live = q4 * 32 < nrows;                              // of the warp
            // values past the last key, up to the product's step of 16: zero, because a zero probability times whatever lay
            // there (NaN, say) would not be
            const int zeros = (it.keys + 15) / 16 * 16 - it.keys;
            if (zeros) {
                unsigned char *const vs = stages + s * stage_bytes + v_at;
                for (int i = st; i < zeros * halves * 8; i += 256) {
                    const int piece = i % (halves * 8);
                    *reinterpret_cast<uint4 *>(vs + (piece >> 3) * 16384 + (it.keys + i / (halves * 8)) * 128 + ((piece & 7) << 4)) =
                        make_uint4(0, 0, 0, 0);
                }
                asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
            }
            ok = mbar_wait(&sh.s_full[u & 1], (u >> 1) & 1);
            if (!__all_sync(0xffffffffu, ok)) { ok = false; break; }
            tc_fence_after();
            if (live) {
                const uint32_t at = tmem + (u & 1) * 128 + lanes;
                uint32_t x[2][32];
                tc_ld32(at + half * 64, x[0]);
                tc_ld32(at + half * 64 + 32, x[1]);
                tc_wait_ld();
                const int mine = it.keys - half * 64;
                if (__any_sync(0xffffffffu, mine < 64)) {
#pragma unroll
                    for (int c = 0; c < 2; ++c)
#pragma unroll
                        for (int j = 0; j < 32; ++j)
                            if (c * 32 + j >= mine) x[c][j] = 0xff800000u;
                }
                float top[4] = {-CUDART_INF_F, -CUDART_INF_F, -CUDART_INF_F, -CUDART_INF_F};
#pragma unroll
                for (int c = 0; c < 2; ++c)
#pragma unroll
                    for (int j = 0; j < 32; j += 2)
                        top[(j >> 1) & 3] = fmax3(top[(j >> 1) & 3], __uint_as_float(x[c][j]), __uint_as_float(x[c][j + 1]));
                // the other half's maximum; past this barrier both have their scores in registers, so that P may overwrite them
                float t = fmaxf(fmaxf(top[0], top[1]), fmaxf(top[2], top[3]));
                sh.top[u & 1][half][r] = t;
                if (!(ok = meet())) break;
                t = fmaxf(t, sh.top[u & 1][half ^ 1][r]);
                const bool above = (t - m) * scale > kTcSlack;
                if (it.fresh) m = t;
                else if (__any_sync(0xffffffffu, above)) {
                    // a maximum well above the reference: O (half of it here) and l move to it
                    ok = mbar_wait(&sh.pv_done[(u - 1) & 1], ((u - 1) >> 1) & 1);
                    if (!__all_sync(0xffffffffu, ok)) { ok = false; break; }
                    tc_fence_after();
                    const float to = above ? t : m, f = to == -CUDART_INF_F ? 1.0f : exp2_fast((m - to) * scale);
                    m = to;
                    l *= f;
#pragma unroll 1
                    for (int c = half * 64; c < min(hd, half * 64 + 64); c += 32) {
                        uint32_t o[32];
                        tc_ld32(tmem + kTcO + lanes + c, o);
                        tc_wait_ld();
#pragma unroll
                        for (int j = 0; j < 32; ++j) o[j] = __float_as_uint(__uint_as_float(o[j]) * f);
                        tc_st32(tmem + kTcO + lanes + c, o);
                    }
                    tc_wait_st();
                }
                const float from = m == -CUDART_INF_F ? 0.0f : m;
                const float2 from2 = make_float2(-from, -from), scale2 = make_float2(scale, scale), shift2 = make_float2(kShift, kShift);
                float sum[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
                for (int c = 0; c < 2; ++c)
#pragma unroll
                    for (int j = 0; j < 32; j += 2) {
                        const float2 d = __ffma2_rn(__fadd2_rn(make_float2(__uint_as_float(x[c][j]), __uint_as_float(x[c][j + 1])), from2), scale2, shift2);
                        const float e = exp2_fast(d.x), f = exp2_fast(d.y);
                        sum[j & 2] += e;
                        sum[(j & 2) + 1] += f;
                        // rounded to the 16-bit type for the product with v; the sum takes the unrounded ones (see probability_base)
                        x[0][c * 16 + j / 2] = D::encode2(e, f);
                    }
                tc_st32(at + half * 32, x[0]);
                l += (sum[0] + sum[1]) + (sum[2] + sum[3]);
                tc_wait_st();
            }
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(&sh.p_ready[u & 1]);
            if (it.leave) {
                if (live) {
                    if (half) sh.sum[r] = l;
                    if (!(ok = meet())) break;
                    if (!half && r < nrows)
                        reinterpret_cast<float2 *>(ws + p.off_pre_ml)[rec + r] = make_float2(__fmul_rn(m, scale) - kShift, l + sh.sum[r]);
                }
                __syncwarp();
                if (lane == 0) mbar_arrive(&sh.item_done[it.item & 3]);
            }
            if (it.stop) break;
            if (++s == nstages) { s = 0; ph ^= 1; }
        }
        if (!ok) {
            if (lane == 0) sh.gave_up[q4] = 1;
            __syncwarp();
            named_bar_arrive(2 + q4, 64);
        }
    } else {
        // -------------------------------------------------------------- Q in, O out: a thread per row
        const int q4 = warp & 3, r = q4 * 32 + lane, G = a.n_heads / a.n_kv;
        const uint32_t lanes = (uint32_t)(q4 * 32) << 16, turn = a.scale < 0.0f ? 0x80008000u : 0u;
        const int items = (tile0 + units + (int)p.pre_tiles - 1) / (int)p.pre_tiles;
        auto bring = [&](int i) {                                           // the rows of Q of this CTA's i'th item
            const int kh = (item0 + i) / p.pre_rt;
            const TcItem x = tc_item(a, p, kh, (item0 + i) % p.pre_rt, cta);
            if (q4 * 32 < x.nrows) {
                const uint32_t row = x.row0 + min(r, x.nrows - 1);
                const uint16_t *src = a.q + (long long)(row / (unsigned)G) * a.ldq + (long long)(kh * G + (int)(row % (unsigned)G)) * hd;
#pragma unroll 1
                for (int c = 0; c < (hd + 15) / 16 * 8; c += 32) {
                    uint32_t x[32];
#pragma unroll
                    for (int j = 0; j < 32; j += 4) {
                        const int d = (c + j) * 2;
                        const uint4 v = d < hd ? *reinterpret_cast<const uint4 *>(src + d) : make_uint4(0, 0, 0, 0);
                        x[j] = v.x ^ turn; x[j + 1] = v.y ^ turn; x[j + 2] = v.z ^ turn; x[j + 3] = v.w ^ turn;
                    }
                    tc_st32(tmem + kTcQ + (i & 1) * 64 + lanes + c, x);
                }
                tc_wait_st();
            }
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(&sh.q_ready[i & 1]);
        };
        bring(0);
        for (int i = 0; i < items; ++i) {
            if (i + 1 < items) bring(i + 1);                                // its buffer was last used by item i - 1, whose O is out
            // (the softmax may be up to two items ahead of this: four barriers)
            ok = mbar_wait(&sh.o_full, i & 1) && mbar_wait(&sh.item_done[i & 3], (i >> 2) & 1);
            if (!__all_sync(0xffffffffu, ok)) { ok = false; break; }
            tc_fence_after();
            const TcItem x = tc_item(a, p, (item0 + i) / p.pre_rt, (item0 + i) % p.pre_rt, cta);
            if (q4 * 32 < x.nrows) {
                float *const dst = reinterpret_cast<float *>(ws + p.off_pre_o) + (x.rec + r) * hd;
#pragma unroll 1
                for (int c = 0; c < hd; c += 32) {
                    uint32_t o[32];
                    tc_ld32(tmem + kTcO + lanes + c, o);
                    tc_wait_ld();
                    if (r < x.nrows)
#pragma unroll
                        for (int j = 0; j < 32; j += 4)
                            if (c + j < hd) *reinterpret_cast<uint4 *>(dst + c + j) = make_uint4(o[j], o[j + 1], o[j + 2], o[j + 3]);
                }
            }
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(&sh.o_free);
        }
    }
    if (!ok && lane == 0 && a.st) atomicAdd(&a.st->wait_timeout, 1ull);
    tc_fence_before();
    __syncthreads();
    if (warp == 1) {
        __syncwarp();
        tc_fence_after();
        tc_dealloc<1>(tmem, 512);
    }
}

template <class D>
static aweq_status tc_launch(const AttentionArgs &a, const AttentionPlan &p, unsigned char *ws, cudaStream_t stream)
{
    CUtensorMap mk, mv;
    aweq_status rc = tma_pool_map(&mk, a.ck, a.n_pages, a.page_size, a.n_kv, a.head_dim, a.page_stride, a.token_stride, a.head_stride, p.box);
    if (rc == AWEQ_OK)
        rc = tma_pool_map(&mv, a.cv, a.n_pages, a.page_size, a.n_kv, a.head_dim, a.page_stride, a.token_stride, a.head_stride, p.box);
    if (rc != AWEQ_OK) return rc;
    static std::atomic<unsigned long long> allowed{0};
    AWEQ_CUDA_OK(allow_smem(attention_tc_kernel<D>, kTcSmem, allowed));
    AWEQ_LAUNCH(attention_tc_kernel<D>, dim3((unsigned)p.tc_ctas), dim3(kTcThreads), kTcSmem, stream, a, p, mk, mv, ws);
    return AWEQ_OK;
}

aweq_status run_attention_tc(const AttentionArgs &a, const AttentionPlan &p, aweq_dtype dt, unsigned char *ws, cudaStream_t stream)
{
    return dt == AWEQ_F16 ? tc_launch<F16>(a, p, ws, stream) : tc_launch<BF16>(a, p, ws, stream);
}

}  // namespace aweq
