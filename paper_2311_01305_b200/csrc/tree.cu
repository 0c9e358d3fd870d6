// aweq_tree_attention: the nodes of drafted trees over a shared prefix, their sequence's keys and the nodes above them.
//
// A node sees all keys of the prefix and all of its sequence before the tree: dense products, for which the rows (node, head)
// that read one key head go together, 128 to a tile.  Of the tree itself it sees what its mask says, mostly a handful of nodes: those
// keys are taken one by one by the launch that joins the parts, which so never touches a key or value that its row does not see.
//
//   S = Q K^T   Q and K in shared memory          -> S in TMEM
//   P = 2^((S - m) scale), a thread to a row, 16-bit, in TMEM over the S it came from
//   O += P V    P in TMEM, V in shared memory     -> O in TMEM
// with the maximum m of a row moving only when a new one exceeds it by more than 8 (a factor of 256), so that O is hardly ever
// rescaled.  Two such sums are under way in a CTA, so that one's products run under the other's exponentials: two row tiles on
// the same keys where a sequence has more than 128 rows to a key head, else the same rows on every other unit of keys.
// A unit is 128 keys (or the whole pages that fit).  The units of all (segment, key head, row tile) items in a row are dealt out evenly
// to a CTA per SM; where a CTA leaves an item it writes a record (m, sum, O of the keys it has seen) for each row and sum.
// Warps: 0 copies keys and values, 1 issues the products, 2 and 3 bring the rows of Q, 4-7 and 8-11 the softmax of the two sums.
#include "tree.cuh"
#include "tensorcore.cuh"

namespace aweq {

constexpr int kTrThreads = 384, kTrQBytes = 64 * 1024, kTrRing = 160 * 1024, kTrMaxTiles = 10;
// registers of a softmax thread and of the others: together no more than the launch gives
constexpr int kTrSoftRegs = 208, kTrOtherRegs = 80;
constexpr float kTrSlack = 8.0f;

struct TreeShared {
    uint64_t full[kTrMaxTiles], empty[kTrMaxTiles], q_ready[2], q_free[2], s_full[2], p_ready[2], pv_done[2], o_free[2];
    uint32_t tmem;
};
constexpr size_t kTrSmem = 1024 + kTrQBytes + kTrRing + sizeof(TreeShared);
static_assert(kTrSmem <= 227 * 1024, "shared memory of a CTA");

static size_t up256(size_t b) { return (b + 255) & ~(size_t)255; }

static TreePlan tree_plan(const aweq_kv_cache *c, long long prefix_len, long long n_seq, long long max_tokens, int max_nodes, int n_heads)
{
    TreePlan p;
    const int G = n_heads / c->n_kv_heads;
    const long long own_rows = (long long)(max_nodes < max_tokens ? max_nodes : max_tokens) * G, pre_rows = max_tokens * G;
    p.two = own_rows > 128;
    p.rows = p.two ? 256 : 128;
    // tiled copies of `box` keys that lie in one page (rows a multiple of eight keep the swizzle's phase)
    p.box = 0;
    if (c->page_size % 8 == 0 && tma_pool_fits(c->page_stride, c->token_stride, c->head_stride)) {
        if (c->page_size <= 128) p.box = c->page_size;
        else if (c->page_size % 128 == 0) p.box = 128;
        else if (c->page_size % 64 == 0) p.box = 64;
    }
    p.unit = p.box ? 128 / p.box * p.box : 128;
    if (p.unit < 96) {
        p.box = 0;
        p.unit = 128;
    }
    p.ctas = kSmCount;
    p.pre_rt = (int)((pre_rows + p.rows - 1) / p.rows);
    p.pre_tiles = (int)((prefix_len + p.unit - 1) / p.unit);
    p.pre_rec = (int)(pre_rows < p.rows ? pre_rows : p.rows);
    p.own_rec = (int)(own_rows < p.rows ? own_rows : p.rows);
    const int sums = p.two ? 1 : 2;
    const long long pre_items = p.pre_tiles ? (long long)c->n_kv_heads * p.pre_rt : 0;
    // (no more row tiles than every sequence's most, nor than the tokens make)
    long long rt = n_seq * ((own_rows + p.rows - 1) / p.rows);
    if (rt > pre_rows / p.rows + n_seq) rt = pre_rows / p.rows + n_seq;
    const size_t pre_kept = p.pre_tiles ? (size_t)(pre_items + p.ctas) * p.pre_rec * sums : 0;
    const size_t own_kept = (size_t)(rt * c->n_kv_heads + p.ctas) * p.own_rec * sums;
    size_t off = up256((size_t)n_seq * sizeof(TreeFirst) + sizeof(TreeTotals));
    p.off_pre_o = off; off += up256(pre_kept * c->head_dim * 4);
    p.off_pre_ml = off; off += up256(pre_kept * 8);
    p.off_own_o = off; off += up256(own_kept * c->head_dim * 4);
    p.off_own_ml = off; off += up256(own_kept * 8);
    p.total = off;
    return p;
}

size_t tree_attention_ws_bytes(const aweq_kv_cache *cache, long long prefix_len, long long max_own, long long n_seq, long long max_tokens,
                               int max_nodes, int n_heads)
{
    (void)max_own;
    return tree_plan(cache, prefix_len, n_seq, max_tokens, max_nodes, n_heads).total;
}

__device__ __forceinline__ AttentionDeal tree_deal(const TreePlan &p, const TreeTotals &t) { return AttentionDeal(t.pre + t.own, p.ctas); }

// A step of one of the two sums: a unit of keys on a row tile.
struct TreeStep {
    int live, fresh, keys;       // rows there; first of its item for this sum in this CTA
};

template <class D>
__global__ void __launch_bounds__(kTrThreads, 1)
tree_units_kernel(const TreeArgs a, const TreePlan p, const __grid_constant__ CUtensorMap mapK, const __grid_constant__ CUtensorMap mapV,
                  unsigned char *ws)
{
    extern __shared__ unsigned char raw[];
    unsigned char *const qs = reinterpret_cast<unsigned char *>((reinterpret_cast<uintptr_t>(raw) + 1023) & ~(uintptr_t)1023);
    unsigned char *const tiles = qs + kTrQBytes;
    TreeShared &sh = *reinterpret_cast<TreeShared *>(tiles + kTrRing);
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, cta = blockIdx.x, hd = a.head_dim;
    const int halves = hd > 64 ? 2 : 1, tile_bytes = halves * 16384, n_tiles = kTrRing / tile_bytes;
    if (tid == 0) {
        for (int i = 0; i < n_tiles; ++i) {
            mbar_init(&sh.full[i], 1);
            mbar_init(&sh.empty[i], 1);
        }
        for (int i = 0; i < 2; ++i) {
            mbar_init(&sh.q_ready[i], 2);
            mbar_init(&sh.q_free[i], 1);
            mbar_init(&sh.s_full[i], 1);
            mbar_init(&sh.p_ready[i], 4);
            mbar_init(&sh.pv_done[i], 1);
            mbar_init(&sh.o_free[i], 4);
        }
        mbar_init_fence();
        if (p.box) {
            tma_prefetch_map(&mapK);
            tma_prefetch_map(&mapV);
        }
    }
    if (warp == 1) tc_alloc<1>(&sh.tmem, 512);
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = sh.tmem;
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    const TreeTotals totals = tree_totals(a, p, ws, cta == 0 && warp == 0);
    if (cta == 0 && tid == 0) *reinterpret_cast<TreeTotals *>(ws + (size_t)a.n_seq * sizeof(TreeFirst)) = totals;
    const AttentionDeal deal = tree_deal(p, totals);
    const long long u0 = cta < deal.ctas ? deal.first(cta) : 0;
    const int units = cta < deal.ctas ? (int)(deal.first(cta + 1) - u0) : 0;
    TreeWalk w;
    if (units) w.begin(a, p, totals, u0);

    bool ok = true;
    if (warp < 4) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kTrOtherRegs));
        if (warp == 0) {
            // ---------------------------------------------------------- copies: a unit's keys, then its values
            int s = 0;
            uint32_t ph = 0;
            if (p.box) {
                const int boxes = p.unit / p.box;
                int page = units && lane < boxes ? w.entry(a, p, lane * p.box) : 0;
                for (int left = units; left > 0; --left) {
                    const int keys = w.keys(p), kh = w.kh, row = (unsigned)(w.tile * p.unit + lane * p.box) % (unsigned)a.page_size;
                    const bool there = lane < boxes && lane * p.box < keys, bad = there && (page < 0 || page >= a.n_pages);
                    const int pid = bad ? 0 : page, n = __popc(__ballot_sync(0xffffffffu, there));
                    if (bad && (w.kh | w.rt | row) == 0 && a.st) atomicAdd(&a.st->out_of_range, 1ull);
                    if (left > 1) {
                        w.advance(a, p);
                        page = lane < boxes ? w.entry(a, p, lane * p.box) : 0;      // the next unit's, while these stages empty
                    }
                    for (int v = 0; v < 2; ++v) {
                        ok = mbar_wait(&sh.empty[s], ph ^ 1);
                        if (!__all_sync(0xffffffffu, ok)) { ok = false; break; }
                        if (lane == 0) mbar_arrive_expect_tx(&sh.full[s], (uint32_t)(n * p.box * 128 * halves));
                        __syncwarp();
                        if (there)
                            for (int h = 0; h < halves; ++h)
                                tma_load4(smem_u32(tiles + s * tile_bytes + h * 16384) + lane * p.box * 128, v ? &mapV : &mapK, h * 64, kh, row, pid,
                                          smem_u32(&sh.full[s]));
                        if (++s == n_tiles) { s = 0; ph ^= 1; }
                    }
                    if (!ok) break;
                }
            } else {
                // pages and strides that tiled copies do not serve: 16 bytes at a time, a tile's under way while the one before lands
                const int per = hd / 8;
                int pending = -1;
                auto landed = [&](int stage) {
                    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                    __syncwarp();
                    if (lane == 0) mbar_arrive(&sh.full[stage]);
                };
                for (int left = units; left > 0; --left) {
                    const int keys = w.keys(p);
                    long long off[4];                           // element of the pool of keys lane, lane + 32, ...; -1: none
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const int r = i * 32 + lane;
                        const int page = w.entry(a, p, r);
                        const unsigned row = (unsigned)(w.tile * p.unit + r) % (unsigned)a.page_size;
                        const bool bad = r < keys && (page < 0 || page >= a.n_pages);
                        if (bad && (w.kh | w.rt) == 0 && (row == 0) && a.st) atomicAdd(&a.st->out_of_range, 1ull);
                        off[i] = r < keys ? (long long)(bad ? 0 : page) * a.page_stride + (long long)row * a.token_stride + w.kh * a.head_stride : -1;
                    }
                    if (left > 1) w.advance(a, p);
                    for (int v = 0; v < 2; ++v) {
                        if (pending >= 0 && !__all_sync(0xffffffffu, mbar_try_wait(&sh.empty[s], ph ^ 1))) {
                            asm volatile("cp.async.wait_group 0;" ::: "memory");
                            landed(pending);
                            pending = -1;
                        }
                        ok = mbar_wait(&sh.empty[s], ph ^ 1);
                        if (!__all_sync(0xffffffffu, ok)) { ok = false; break; }
                        const uint16_t *const pool = v ? a.cv : a.ck;
                        const uint32_t dst = smem_u32(tiles + s * tile_bytes);
#pragma unroll
                        for (int i = 0; i < 4; ++i)
                            for (int c = 0; c < halves * 8; ++c) {
                                const int r = i * 32 + lane;
                                const bool in = off[i] >= 0 && c < per;
                                asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst + (c >> 3) * 16384 + r * 128 + (((c ^ r) & 7) << 4)),
                                             "l"(pool + (in ? off[i] + c * 8 : 0)), "r"(in ? 16 : 0) : "memory");
                            }
                        asm volatile("cp.async.commit_group;" ::: "memory");
                        if (pending >= 0) {
                            asm volatile("cp.async.wait_group 1;" ::: "memory");
                            landed(pending);
                        }
                        pending = s;
                        if (++s == n_tiles) { s = 0; ph ^= 1; }
                    }
                    if (!ok) break;
                }
                asm volatile("cp.async.wait_group 0;" ::: "memory");
                if (pending >= 0) landed(pending);
            }
            if (!ok)                                            // gave up: let what is under way land (bounded) before the memory goes
                for (int i = 0; i < n_tiles; ++i) mbar_wait(&sh.full[i], ph ^ (i >= s ? 1u : 0u));
        } else if (warp == 1) {
            // ---------------------------------------------------------- products
            const bool lead = tc_elect();
            const uint32_t idesc_s = tc_idesc_f16(D::kBf16, 128, 128, false), idesc_o = tc_idesc_f16(D::kBf16, 128, (hd + 15) / 16 * 16, true);
            const int ksteps = (hd + 15) / 16, steps = units << p.two;
            // the stages of the next K and V tiles (every other one)
            int ks = 0, vs = 1, item = 0, of_item = 0, unit = 0;     // item: its number here; of_item: units of it so far
            uint32_t kph = 0, vph = 0, cnt[2] = {0, 0}, outs[2] = {0, 0};
            TreeStep st[2];
            bool have_unit = false;
            // S of step j; the walk goes on with the last step of a unit
            auto scores = [&](int j) {
                TreeStep &x = st[j & 1];
                x.live = p.two ? w.rows(a, p) > (j & 1) * 128 : 1;
                x.fresh = p.two ? of_item == 0 : of_item < 2;
                x.keys = w.keys(p);
                const int buf = p.two ? 0 : item & 1;
                if (of_item == 0 && !have_unit) {
                    if (!mbar_wait(&sh.q_ready[buf], (p.two ? item : item >> 1) & 1)) return false;
                }
                if (!have_unit && !mbar_wait(&sh.full[ks], kph)) return false;
                have_unit = true;
                const bool last = !p.two || (j & 1);
                if (x.live) {
                    tc_fence_after();
                    const uint32_t q = tc_desc(smem_u32(qs) + (p.two ? j & 1 : buf) * 32768), k = tc_desc(smem_u32(tiles) + ks * tile_bytes);
#pragma unroll
                    for (int i = 0; i < 8; ++i)
                        if (i < ksteps)
                            tc_mma_f16_ss(tmem + (j & 1) * 128, q + (i >> 2) * 1024 + 2 * (i & 3), k + (i >> 2) * 1024 + 2 * (i & 3), idesc_s, i > 0, lead);
                    tc_commit<1>(&sh.s_full[j & 1], lead);
                }
                if (last) {
                    tc_commit<1>(&sh.empty[ks], lead);
                    ks += 2;
                    if (ks >= n_tiles) { ks -= n_tiles; kph ^= 1; }
                    have_unit = false;
                    ++unit;
                    ++of_item;
                    if (unit == units || w.tile + 1 == w.tiles) {
                        tc_commit<1>(&sh.q_free[buf], lead);
                        ++item;
                        of_item = 0;
                    }
                    if (unit < units) w.advance(a, p);
                }
                return true;
            };
            for (int j = 0; ok && j < 2 && j < steps; ++j) ok = scores(j);
            for (int j = 0; ok && j < steps; ++j) {
                const int s = j & 1;
                const TreeStep x = st[s];
                if (x.live) {
                    if (!(ok = mbar_wait(&sh.full[vs], vph) && mbar_wait(&sh.p_ready[s], cnt[s] & 1))) break;
                    ++cnt[s];
                    if (x.fresh && outs[s]++ > 0 && !(ok = mbar_wait(&sh.o_free[s], outs[s] & 1))) break;
                    tc_fence_after();
                    const uint32_t v = tc_desc_mn(smem_u32(tiles) + vs * tile_bytes, 16384);
                    const int n = (x.keys + 15) / 16;
#pragma unroll
                    for (int i = 0; i < 8; ++i)
                        if (i < n) tc_mma_f16_ta(tmem + 256 + s * 128, tmem + s * 128 + i * 8, v + i * 128, idesc_o, !x.fresh || i > 0, lead);
                    tc_commit<1>(&sh.pv_done[s], lead);
                }
                if (!p.two || s) {
                    tc_commit<1>(&sh.empty[vs], lead);
                    vs += 2;
                    if (vs >= n_tiles) { vs -= n_tiles; vph ^= 1; }
                }
                if (j + 2 < steps) ok = scores(j + 2);
            }
        } else {
            // ---------------------------------------------------------- the rows of Q, half of them to a warp
            const int G = a.n_heads / a.n_kv, bufs = p.two ? 1 : 2, per = p.rows / 2;
            const uint32_t turn = a.scale < 0.0f ? 0x80008000u : 0u;
            int item = 0;
            for (int u = 0; u < units; ++item) {
                const int buf = item % bufs;
                if (item >= bufs) ok = mbar_wait(&sh.q_free[buf], (item / bufs - 1) & 1);
                if (!__all_sync(0xffffffffu, ok)) { ok = false; break; }
                const int rows = w.rows(a, p), r0 = (warp - 2) * per;
                // a lane takes a 16-byte piece of every other row
                const int c = lane & 15;
                if (c < halves * 8)
                    for (int r = r0 + (lane >> 4); r < min(r0 + per, (rows + 31) & ~31); r += 16) {
                        uint4 v[8];
#pragma unroll
                        for (int i = 0; i < 8; ++i) {
                            const int rr = r + 2 * i;
                            v[i] = make_uint4(0, 0, 0, 0);
                            if (rr < rows && rr < r0 + per && c * 8 < hd) {
                                const unsigned row = (unsigned)(w.rt * p.rows + rr);
                                const uint16_t *src = a.q + (long long)(w.t0 + (int)(row / (unsigned)G)) * a.ldq + (long long)(w.kh * G + (int)(row % (unsigned)G)) * hd;
                                v[i] = *reinterpret_cast<const uint4 *>(src + c * 8);
                            }
                        }
#pragma unroll
                        for (int i = 0; i < 8; ++i) {
                            const int rr = r + 2 * i;
                            if (rr < r0 + per)
                                *reinterpret_cast<uint4 *>(qs + (p.two ? rr >> 7 : buf) * 32768 + (c >> 3) * 16384 + (rr & 127) * 128 + (((c ^ rr) & 7) << 4)) =
                                    make_uint4(v[i].x ^ turn, v[i].y ^ turn, v[i].z ^ turn, v[i].w ^ turn);
                        }
                    }
                asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                __syncwarp();
                if (lane == 0) mbar_arrive(&sh.q_ready[buf]);
                // on to the next item
                const int rest = min(w.tiles - w.tile, units - u);
                u += rest;
                if (u < units) {
                    w.tile = w.tiles - 1;
                    w.advance(a, p);
                }
            }
        }
    } else {
        // -------------------------------------------------------------- softmax: a thread to a row
        asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kTrSoftRegs));
        const int sum = (warp - 4) >> 2, q4 = warp & 3, r = q4 * 32 + lane;
        const uint32_t at = tmem + sum * 128 + ((uint32_t)(q4 * 32) << 16), acc = at + 256;
        // a negative scale turned q's signs; a zero one must leave -inf where a key is not seen
        const float scale = (a.scale == 0.0f ? 1.17549435e-38f : fabsf(a.scale)) * 1.4426950408889634f;
        constexpr float kShift = D::kBf16 ? 0.0f : kProbabilityShift;
        uint32_t cnt = 0;
        int of_item = 0, taken = 0;                             // units of the item so far, and those of this sum
        float m = -CUDART_INF_F, l = 0.0f;
        for (int u = 0; u < units; ++u) {
            const int rows = w.rows(a, p), mine = rows - (p.two ? sum * 128 : 0), keys = w.keys(p);
            const bool leave = u + 1 == units || w.tile + 1 == w.tiles;
            if (mine > 0 && (p.two || (u & 1) == sum)) {
                const bool fresh = taken == 0, live = q4 * 32 < mine;
                ++taken;
                // values past the last key, up to the product's step of 16: zero, because a zero probability times whatever lay
                // there (NaN, say) would not be
                const int zeros = (keys + 15) / 16 * 16 - keys;
                if (zeros && (!p.two || sum == 0)) {
                    const int t = 2 * u + 1, stage = t % n_tiles;
                    ok = mbar_wait(&sh.full[stage], (t / n_tiles) & 1);
                    if (!__all_sync(0xffffffffu, ok)) { ok = false; break; }
                    unsigned char *const vt = tiles + stage * tile_bytes;
                    for (int i = r; i < zeros * halves * 8; i += 128) {
                        const int piece = i % (halves * 8);
                        *reinterpret_cast<uint4 *>(vt + (piece >> 3) * 16384 + (keys + i / (halves * 8)) * 128 + ((piece & 7) << 4)) = make_uint4(0, 0, 0, 0);
                    }
                    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                }
                ok = mbar_wait(&sh.s_full[sum], cnt & 1);
                if (!__all_sync(0xffffffffu, ok)) { ok = false; break; }
                tc_fence_after();
                if (live) {
                    uint32_t x[4][32];
#pragma unroll
                    for (int c = 0; c < 4; ++c) tc_ld32(at + c * 32, x[c]);
                    tc_wait_ld();
                    if (keys < 128)
#pragma unroll
                        for (int c = 0; c < 4; ++c)
#pragma unroll
                            for (int j = 0; j < 32; ++j)
                                if (c * 32 + j >= keys) x[c][j] = 0xff800000u;
                    float top[4] = {-CUDART_INF_F, -CUDART_INF_F, -CUDART_INF_F, -CUDART_INF_F};
#pragma unroll
                    for (int c = 0; c < 4; ++c)
#pragma unroll
                        for (int j = 0; j < 32; j += 2) top[(j >> 1) & 3] = fmax3(top[(j >> 1) & 3], __uint_as_float(x[c][j]), __uint_as_float(x[c][j + 1]));
                    const float t = fmaxf(fmaxf(top[0], top[1]), fmaxf(top[2], top[3]));
                    const bool above = (t - m) * scale > kTrSlack;
                    if (fresh) {
                        m = t;
                        l = 0.0f;
                    } else if (__any_sync(0xffffffffu, above)) {
                        // a maximum well above the reference: O and l move to it
                        ok = mbar_wait(&sh.pv_done[sum], (cnt - 1) & 1);
                        if (!__all_sync(0xffffffffu, ok)) { ok = false; break; }
                        tc_fence_after();
                        const float to = above ? t : m, f = to == -CUDART_INF_F ? 1.0f : exp2_fast((m - to) * scale);
                        m = to;
                        l *= f;
#pragma unroll 1
                        for (int c = 0; c < hd; c += 16) {
                            uint32_t o[16];
                            tc_ld16(acc + c, o);
                            tc_wait_ld();
#pragma unroll
                            for (int j = 0; j < 16; ++j) o[j] = __float_as_uint(__uint_as_float(o[j]) * f);
                            tc_st16(acc + c, o);
                        }
                        tc_wait_st();
                    }
                    const float from = m == -CUDART_INF_F ? 0.0f : m;
                    const float2 from2 = make_float2(-from, -from), scale2 = make_float2(scale, scale), shift2 = make_float2(kShift, kShift);
                    float part[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
                    for (int c = 0; c < 4; ++c)
#pragma unroll
                        for (int j = 0; j < 32; j += 2) {
                            const float2 d = __ffma2_rn(__fadd2_rn(make_float2(__uint_as_float(x[c][j]), __uint_as_float(x[c][j + 1])), from2), scale2, shift2);
                            const float e = exp2_fast(d.x), f = exp2_fast(d.y);
                            part[j & 2] += e;
                            part[(j & 2) + 1] += f;
                            // rounded to the 16-bit type for the product with v; the sum takes the unrounded ones (see probability_base)
                            x[c >> 1][(c & 1) * 16 + j / 2] = D::encode2(e, f);
                        }
                    tc_st32(at, x[0]);
                    tc_st32(at + 32, x[1]);
                    l += (part[0] + part[1]) + (part[2] + part[3]);
                    tc_wait_st();
                }
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(&sh.p_ready[sum]);
                ++cnt;
            }
            ++of_item;
            if (leave) {
                const int own_rec = w.own ? p.own_rec : p.pre_rec, stride = p.two ? own_rec : 2 * own_rec;
                const long long rec = (long long)(w.item + cta) * stride + (p.two ? sum * 128 : sum * own_rec) + r;
                float2 *const ml = reinterpret_cast<float2 *>(ws + (w.own ? p.off_own_ml : p.off_pre_ml));
                if (taken) {
                    ok = mbar_wait(&sh.pv_done[sum], (cnt - 1) & 1);
                    if (!__all_sync(0xffffffffu, ok)) { ok = false; break; }
                    tc_fence_after();
                    if (q4 * 32 < mine) {
                        float *const dst = reinterpret_cast<float *>(ws + (w.own ? p.off_own_o : p.off_pre_o)) + rec * hd;
#pragma unroll 1
                        for (int c = 0; c < hd; c += 32) {
                            uint32_t o[32];
                            tc_ld32(acc + c, o);
                            tc_wait_ld();
                            if (r < mine)
#pragma unroll
                                for (int j = 0; j < 32; j += 4)
                                    if (c + j < hd) *reinterpret_cast<uint4 *>(dst + c + j) = make_uint4(o[j], o[j + 1], o[j + 2], o[j + 3]);
                        }
                        if (r < mine) ml[rec] = make_float2(m == -CUDART_INF_F ? m : __fmul_rn(m, scale) - kShift, l);
                    }
                    tc_fence_before();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(&sh.o_free[sum]);
                } else if (!p.two && r < mine)
                    ml[rec] = make_float2(-CUDART_INF_F, 0.0f);         // the item had no unit for this sum
                of_item = taken = 0;
            }
            if (u + 1 < units) w.advance(a, p);
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

// ------------------------------------------------------------------ the tree itself, and the join
// A warp per row.  Its halves take turns at the visible nodes and the records, 16 lanes with eight dims each; binary32 throughout.
template <class D>
__global__ void __launch_bounds__(128)
tree_join_kernel(const TreeArgs a, const TreePlan p, const unsigned char *__restrict__ ws)
{
    pdl_begin();
    const int lane = threadIdx.x & 31, half = lane >> 4, d0 = (lane & 15) * 8, hd = a.head_dim, G = a.n_heads / a.n_kv;
    const unsigned row = blockIdx.x * 4 + (threadIdx.x >> 5);
    const int tok = (int)(row / (unsigned)a.n_heads), h = (int)(row % (unsigned)a.n_heads), kh = h / G;
    const TreeTotals totals = *reinterpret_cast<const TreeTotals *>(ws + (size_t)a.n_seq * sizeof(TreeFirst));
    if (tok >= totals.tokens) return;
    // the last sequence that starts at or before the token (32 at a time)
    int b = 0;
    for (int n = a.n_seq; n > 1;) {
        const int step = (n + 31) / 32, at = b + lane * step;
        const bool before = lane * step < n && __ldg(a.start + at) <= tok;
        const int k = 31 - __clz(__ballot_sync(0xffffffffu, before) | 1u);
        b += k * step;
        n = min(step, n - k * step);
    }
    const TreeSeq s = tree_load(a, b);
    const int node = tok - s.t0;
    if (node < 0 || node >= s.nodes) return;                    // (more nodes than there may be: counted, not computed)
    const float scale = a.scale * 1.4426950408889634f;
    const bool in = d0 < hd;
    float m = -CUDART_INF_F, l = 0.0f, o[8] = {};
    // ---- records
    const AttentionDeal deal = tree_deal(p, totals);
    auto records = [&](const float *ro, const float2 *rml, long long first, int rec_rows, int in_rec, long long unit0, int n_units) {
        const int c0 = deal.cta_of(unit0), c1 = deal.cta_of(unit0 + n_units - 1), sums = p.two ? 1 : 2;
        for (int i = half; i < (c1 - c0 + 1) * sums; i += 2) {
            const long long rec = ((first + c0 + i / sums) * sums + i % sums) * rec_rows + in_rec;
            const float2 x = rml[rec];
            if (x.x == -CUDART_INF_F && x.y == 0.0f) continue;  // (its output may be anything)
            float4 v0 = make_float4(0, 0, 0, 0), v1 = v0;
            if (in) {
                v0 = *reinterpret_cast<const float4 *>(ro + rec * hd + d0);
                v1 = *reinterpret_cast<const float4 *>(ro + rec * hd + d0 + 4);
            }
            const float to = fmaxf(m, x.x), f = m == -CUDART_INF_F ? 0.0f : exp2_fast(m - to), g = exp2_fast(x.x - to);
            m = to;
            l = l * f + x.y * g;
            const float v[8] = {v0.x, v0.y, v0.z, v0.w, v1.x, v1.y, v1.z, v1.w};
#pragma unroll
            for (int j = 0; j < 8; ++j) o[j] = o[j] * f + v[j] * g;
        }
    };
    if (p.pre_tiles) {
        const unsigned in_all = (unsigned)(tok * G + h % G), rt = in_all / (unsigned)p.rows;
        const long long item = (long long)kh * tree_tiles(totals.tokens * G, p.rows) + rt;
        records(reinterpret_cast<const float *>(ws + p.off_pre_o), reinterpret_cast<const float2 *>(ws + p.off_pre_ml), item, p.pre_rec,
                (int)(in_all - rt * p.rows), item * p.pre_tiles, p.pre_tiles);
    }
    if (s.ctx) {
        const TreeFirst f = reinterpret_cast<const TreeFirst *>(ws)[b];
        const unsigned in_seq = (unsigned)(node * G + h % G), rt = in_seq / (unsigned)p.rows;
        const int within = kh * tree_tiles(s.nodes * G, p.rows) + (int)rt;
        records(reinterpret_cast<const float *>(ws + p.off_own_o), reinterpret_cast<const float2 *>(ws + p.off_own_ml), f.item + within, p.own_rec,
                (int)(in_seq - rt * p.rows), totals.pre + f.unit + (long long)within * f.tiles, f.tiles);
    }
    // ---- the nodes that this one sees
    float q[8] = {};
    if (in) widen8<D>(*reinterpret_cast<const uint4 *>(a.q + (long long)tok * a.ldq + (long long)h * hd + d0), q);
    // a page that is none counts where its first key is
    if (h == 0 && lane == 0 && s.base + node >= 0 && (unsigned)(s.base + node) % (unsigned)a.page_size == 0 && a.st) {
        const int page = __ldg(a.page_table + (long long)b * a.ld_table + (unsigned)(s.base + node) / (unsigned)a.page_size);
        if (page < 0 || page >= a.n_pages) atomicAdd(&a.st->out_of_range, 1ull);
    }
    bool any = false;
    for (int word = 0; word < a.words; ++word) {
        unsigned long long bits = (unsigned long long)__ldg(a.mask + (long long)tok * a.words + word);
        const int left = s.nodes - word * 64;
        if (left <= 0) break;
        if (left < 64) bits &= (1ull << left) - 1;
        // (a length below the number of nodes: the first have no key)
        const int gone = -s.base - word * 64;
        if (gone > 0) bits &= gone < 64 ? ~0ull << gone : 0ull;
        any |= bits != 0;
        while (bits) {
            // two nodes, one to each half
            const int n0 = __ffsll((long long)bits) - 1;
            bits &= bits - 1;
            const int n1 = bits ? __ffsll((long long)bits) - 1 : -1;
            bits &= bits ? bits - 1 : 0;
            const int n = half ? n1 : n0, key = s.base + word * 64 + n;
            float sc = 0.0f, v[8] = {};
            if (n >= 0) {
                const unsigned pg = (unsigned)key / (unsigned)a.page_size;
                int page = __ldg(a.page_table + (long long)b * a.ld_table + pg);
                if (page < 0 || page >= a.n_pages) page = 0;
                const long long at = (long long)page * a.page_stride + (long long)(key - (int)pg * a.page_size) * a.token_stride + kh * a.head_stride + d0;
                if (in) {
                    float k[8];
                    widen8<D>(*reinterpret_cast<const uint4 *>(a.ck + at), k);
                    widen8<D>(*reinterpret_cast<const uint4 *>(a.cv + at), v);
#pragma unroll
                    for (int j = 0; j < 8; ++j) sc = __fmaf_rn(q[j], k[j], sc);
                }
            }
#pragma unroll
            for (int x = 8; x > 0; x >>= 1) sc += __shfl_xor_sync(0xffffffffu, sc, x);
            sc = n >= 0 ? sc * scale : -CUDART_INF_F;
            if (n < 0) continue;
            const float to = sc != sc ? sc : fmaxf(m, sc), base = to == -CUDART_INF_F ? 0.0f : to;
            const float f = exp2_fast(m - base), g = exp2_fast(sc - base);
            m = to;
            l = l * f + g;
#pragma unroll
            for (int j = 0; j < 8; ++j) o[j] = o[j] * f + v[j] * g;
        }
    }
    // ---- the halves together
    const float m1 = __shfl_xor_sync(0xffffffffu, m, 16), l1 = __shfl_xor_sync(0xffffffffu, l, 16);
    const float to = fmaxf(m, m1), base = to == -CUDART_INF_F ? 0.0f : to, f = exp2_fast(m - base), g = exp2_fast(m1 - base);
    l = l * f + l1 * g;
    const bool none = !any && s.ctx == 0 && a.prefix_len == 0;
    const float inv = none ? 0.0f : 1.0f / l;
#pragma unroll
    for (int j = 0; j < 8; ++j) o[j] = none ? 0.0f : (o[j] * f + __shfl_xor_sync(0xffffffffu, o[j], 16) * g) * inv;
    if (in && half == 0)
        *reinterpret_cast<uint4 *>(a.out + (long long)tok * a.ldo + (long long)h * hd + d0) =
            make_uint4(D::encode2(o[0], o[1]), D::encode2(o[2], o[3]), D::encode2(o[4], o[5]), D::encode2(o[6], o[7]));
}

template <class D>
static aweq_status tree_launch(const TreeArgs &a, const TreePlan &p, unsigned char *ws, cudaStream_t stream)
{
    CUtensorMap mk = {}, mv = {};
    if (p.box) {
        aweq_status rc = tma_pool_map(&mk, a.ck, a.n_pages, a.page_size, a.n_kv, a.head_dim, a.page_stride, a.token_stride, a.head_stride, p.box);
        if (rc == AWEQ_OK)
            rc = tma_pool_map(&mv, a.cv, a.n_pages, a.page_size, a.n_kv, a.head_dim, a.page_stride, a.token_stride, a.head_stride, p.box);
        if (rc != AWEQ_OK) return rc;
    }
    static std::atomic<unsigned long long> allowed{0};
    AWEQ_CUDA_OK(allow_smem(tree_units_kernel<D>, kTrSmem, allowed));
    AWEQ_LAUNCH(tree_units_kernel<D>, dim3((unsigned)p.ctas), dim3(kTrThreads), kTrSmem, stream, a, p, mk, mv, ws);
    const long long rows = (long long)a.max_tokens * a.n_heads;
    AWEQ_LAUNCH(tree_join_kernel<D>, dim3((unsigned)((rows + 3) / 4)), dim3(128), 0, stream, a, p, (const unsigned char *)ws);
    return AWEQ_OK;
}

aweq_status run_tree_attention(const TreeArgs &a, const aweq_kv_cache *cache, void *ws, cudaStream_t stream)
{
    const TreePlan p = tree_plan(cache, a.prefix_len, a.n_seq, a.max_tokens, a.max_nodes, a.n_heads);
    unsigned char *const w = reinterpret_cast<unsigned char *>(ws);
    return cache->dt == AWEQ_F16 ? tree_launch<F16>(a, p, w, stream) : tree_launch<BF16>(a, p, w, stream);
}

}  // namespace aweq
