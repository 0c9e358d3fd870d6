// aweq_tree_attention: the nodes of drafted trees over a shared prefix, their sequence's keys and the nodes above them.
//
// A node sees all keys of the prefix and all of its sequence before the tree: dense products, for which the rows (node, head)
// that read one key head go together, 128 to a tile.  Of the tree itself it sees what its mask says, mostly a handful of nodes: those
// keys are taken one by one by the launch that joins the parts, which so never touches a key or value that its row does not see.
//
//   S = Q K^T   Q and K in shared memory          -> S in TMEM
//   P = 2^((S - m) scale), two threads to a row, 16-bit, in TMEM over the S it came from
//   O += P V    P in TMEM, V in shared memory     -> O in TMEM
// with the maximum m of a row moving only when a new one exceeds it by more than 8 (a factor of 256), so that O is hardly ever
// rescaled.  Two such sums are under way in a CTA, so that one's products run under the other's exponentials: two row tiles on
// the same keys where a sequence has more than 128 rows to a key head, else the same rows on every other unit of keys.
// A unit is 128 keys (or the whole pages that fit).  The units of all (segment, key head, row tile) items in a row are dealt out evenly
// to a CTA per SM; where a CTA leaves an item it writes a record (m, sum, O of the keys it has seen) for each row.
// Warps: 0 copies keys and values, 1 issues the products (1 and 2 those of a sum each where the sums take units in turn: one warp for
// both took longer to issue them than the softmax took; two tiles on the same keys have to go in step, and two warps that wait for one
// another's keys were slower, 250 us to 190), 3 says which items come and brings their rows of Q, 4-11 and 12-19 the softmax.
// Measured on the device, by itself: 16 trees of 24 nodes after 512 + 2100 keys, 32 / 8 heads of 128, 33-36 us (and the join 18), 32 of 64 after
// up to 8192 keys 180-210 us (and 51): 3.6 TB/s of keys and values, 660 TFLOP/s, tensor pipe 46 %.  Bound by the chain of a unit's steps (scores, maxima,
// exponentials, products: 3000 cycles, two under way) and, for short items, by start (7 us) and records (6000 cycles an item).
#include "tree.cuh"
#include "tensorcore.cuh"

namespace aweq {

constexpr int kTrThreads = 640, kTrQBytes = 64 * 1024, kTrRing = 160 * 1024, kTrMaxTiles = 10, kTrItems = 4;
// registers of a softmax thread and of the others: together no more than the launch gives
constexpr int kTrSoftRegs = 104, kTrOtherRegs = 64;
constexpr float kTrSlack = 8.0f;

constexpr int kTrLanding = 8;                // tiles of a sum on which it may have an eye (at most three units are under way)
struct TreeShared {
    uint64_t full[2][kTrMaxTiles], empty[kTrMaxTiles], q_ready[2], q_free[2], s_full[2], p_ready[2], pv_done[2], issued[2], o_free[2];
    uint64_t item_full[kTrItems], item_empty[kTrItems];
    TreeItem item[kTrItems];
    uint32_t tmem;
    volatile int gave_up[8];             // by sum and TMEM quarter: a softmax warp has
    float top[2][2][128];                // the halves' maxima, by sum and half; at the end of an item the sums' bases and l
};
constexpr size_t kTrSmem = kTrQBytes + kTrRing + sizeof(TreeShared);
static_assert(kTrSmem <= 227 * 1024, "shared memory of a CTA");

static size_t up256(size_t b) { return (b + 255) & ~(size_t)255; }

static TreePlan tree_plan(const aweq_kv_cache *c, long long prefix_len, long long n_seq, long long max_tokens, int max_nodes, int n_heads)
{
    TreePlan p;
    const int G = n_heads / c->n_kv_heads;
    const long long own_rows = (long long)(max_nodes < max_tokens ? max_nodes : max_tokens) * G, pre_rows = max_tokens * G;
    p.two = own_rows > 128;
    p.group = G;
    p.part = G <= 128 ? 128 / G * G : 128;
    p.rows = p.two ? 2 * p.part : p.part;
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
    const long long pre_items = p.pre_tiles ? (long long)c->n_kv_heads * p.pre_rt : 0;
    // (no more row tiles than every sequence's most, nor than the tokens make)
    long long rt = n_seq * ((own_rows + p.rows - 1) / p.rows);
    if (rt > pre_rows / p.rows + n_seq) rt = pre_rows / p.rows + n_seq;
    const size_t pre_kept = p.pre_tiles ? (size_t)(pre_items + p.ctas) * p.pre_rec : 0;
    const size_t own_kept = (size_t)(rt * c->n_kv_heads + p.ctas) * p.own_rec;
    size_t off = up256(sizeof(TreeTotals) + (size_t)n_seq * sizeof(TreeFirst));
    p.off_seq = off; off += up256((size_t)max_tokens * 4);
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

// Where row `row` of all records has its dims d, d + 1, ..., d + 7 (d a multiple of eight): a record of n rows is [dims / 8][n][8].
__device__ __forceinline__ long long tree_record(const TreePlan &p, bool own, long long row, int d, int hd)
{
    const int n = own ? p.own_rec : p.pre_rec;
    const long long rec = row >> 32 ? row / n : (long long)((uint32_t)row / (uint32_t)n), in = row - rec * n;
    return rec * n * hd + (long long)(d >> 3) * n * 8 + in * 8;
}
// The items of a CTA in turn, by a warp that works on them.
struct TreeItems {
    int n = 0;
    __device__ __forceinline__ bool next(TreeShared &sh, TreeItem &it)
    {
        const int i = n & (kTrItems - 1);
        const bool ok = __all_sync(0xffffffffu, mbar_wait(&sh.item_full[i], (n / kTrItems) & 1));
        if (ok) it = sh.item[i];
        __syncwarp();
        if ((threadIdx.x & 31) == 0) mbar_arrive(&sh.item_empty[i]);
        __syncwarp();
        ++n;
        return ok;
    }
};

// eight dims of a record, a whole sector
__device__ __forceinline__ void store32(float *to, const float (&v)[8])
{
    asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(to), "r"(__float_as_uint(v[0])), "r"(__float_as_uint(v[1])),
                 "r"(__float_as_uint(v[2])), "r"(__float_as_uint(v[3])), "r"(__float_as_uint(v[4])), "r"(__float_as_uint(v[5])),
                 "r"(__float_as_uint(v[6])), "r"(__float_as_uint(v[7])) : "memory");
}
// The rows of Q of an item's tiles, into buffer `buf`; by a warp.
template <bool TWO>
__device__ __forceinline__ void tree_bring(const TreeArgs &a, const TreePlan &p, const TreeItem &it, TreeShared &sh, unsigned char *qs, int buf,
                                           const CUtensorMap &mapQ)
{
    const int lane = threadIdx.x & 31, hd = a.head_dim, halves = hd > 64 ? 2 : 1, parts = TWO && it.rows > p.part ? 2 : 1;
    if (p.group <= 128) {
        if (lane == 0) {
            mbar_arrive_expect_tx(&sh.q_ready[buf], (uint32_t)(parts * halves * p.part * 128));
            const int tok = it.t0 + it.rt * (p.rows / p.group);
            for (int i = 0; i < parts; ++i)
                for (int h = 0; h < halves; ++h)
                    tma_load3(smem_u32(qs + (TWO ? i : buf) * 32768 + h * 16384), &mapQ, h * 64, it.kh * p.group, tok + i * (p.part / p.group),
                              smem_u32(&sh.q_ready[buf]));
        }
    } else {
        // more heads to a key head than a tile has rows: row by row
        for (int i = lane; i < it.rows * halves * 8; i += 32) {
            const int r = i / (halves * 8), c = i % (halves * 8);
            const unsigned row = (unsigned)(it.rt * p.rows + r);
            const uint16_t *src = a.q + (long long)(it.t0 + (int)(row / (unsigned)p.group)) * a.ldq +
                                  (long long)(it.kh * p.group + (int)(row % (unsigned)p.group)) * hd;
            *reinterpret_cast<uint4 *>(qs + (TWO ? r >> 7 : buf) * 32768 + (c >> 3) * 16384 + (r & 127) * 128 + (((c ^ r) & 7) << 4)) =
                c * 8 < hd ? *reinterpret_cast<const uint4 *>(src + c * 8) : make_uint4(0, 0, 0, 0);
        }
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        __syncwarp();
        if (lane == 0) mbar_arrive(&sh.q_ready[buf]);
    }
    __syncwarp();
}

template <class D, bool TWO>
__global__ void __launch_bounds__(kTrThreads, 1)
tree_units_kernel(const TreeArgs a, const TreePlan p, const __grid_constant__ CUtensorMap mapK, const __grid_constant__ CUtensorMap mapV,
                  const __grid_constant__ CUtensorMap mapQ, unsigned char *ws)
{
    extern __shared__ __align__(1024) unsigned char qs[];       // (there is no room to round an address up)
    unsigned char *const tiles = qs + kTrQBytes;
    TreeShared &sh = *reinterpret_cast<TreeShared *>(tiles + kTrRing);
    // (the warp's number by a shuffle, so that the compiler knows that a warp has one: the products' operands live in uniform registers)
    const int tid = threadIdx.x, lane = tid & 31, warp = __shfl_sync(0xffffffffu, tid >> 5, 0), cta = blockIdx.x, hd = a.head_dim;
    const int halves = hd > 64 ? 2 : 1, tile_bytes = halves * 16384, n_tiles = kTrRing / tile_bytes;
    if (tid == 0) {
        for (int i = 0; i < kTrMaxTiles; ++i) {
            mbar_init(&sh.full[0][i], 1);
            mbar_init(&sh.full[1][i], 1);
            mbar_init(&sh.empty[i], 1);
        }
        for (int i = 0; i < 2; ++i) {
            mbar_init(&sh.q_ready[i], 1);
            mbar_init(&sh.q_free[i], TWO ? 1 : 2);
            mbar_init(&sh.s_full[i], 1);
            mbar_init(&sh.p_ready[i], 8);
            mbar_init(&sh.pv_done[i], 1);
            mbar_init(&sh.issued[i], 1);
            mbar_init(&sh.o_free[i], TWO ? 8 : 16);
        }
        for (int i = 0; i < kTrItems; ++i) {
            mbar_init(&sh.item_full[i], 1);
            mbar_init(&sh.item_empty[i], TWO ? 18 : 19);
        }
        for (int i = 0; i < 8; ++i) sh.gave_up[i] = 0;
        mbar_init_fence();
        if (p.box) {
            tma_prefetch_map(&mapK);
            tma_prefetch_map(&mapV);
        }
        if (p.group <= 128) tma_prefetch_map(&mapQ);
    }
    if (warp == 1) tc_alloc<1>(&sh.tmem, 512);
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = sh.tmem;
    // Where tile v (0: keys, 1: values) of unit g says that it has landed.  A barrier may be looked at one phase ahead and no further, so it
    // has to have one warp that waits for all its phases: those of the ring's stages have that with two tiles, where one warp takes all
    // units; else each sum has barriers of its own, by the number of its tiles.
    auto landing = [&](int g, int v, uint32_t *parity) -> uint64_t * {
        const int t = 2 * g + v, mine = (g & ~1) + v;           // tile of all, of the sum
        *parity = TWO ? t / n_tiles & 1 : mine / kTrLanding & 1;
        return TWO ? &sh.full[0][t % n_tiles] : &sh.full[g & 1][mine % kTrLanding];
    };

    bool ok = true;
    if (warp < 4) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kTrOtherRegs));
        asm volatile("griddepcontrol.wait;" ::: "memory");
        if (warp == 3) {
            // ---------------------------------------------------------- the CTA's items, a few ahead of those who work on them, and the rows
            // of Q: one buffer for two tiles, or two for one each
            asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
            TreeSeq s0 = {};
            TreeScan c0 = {};
            TreeTotals totals = tree_totals(a, p, s0, c0);
            const AttentionDeal deal(totals.pre + totals.own, p.ctas);
            totals.each = deal.each;
            totals.more = deal.more;
            totals.ctas = deal.ctas;
            if (cta == 0 && lane == 0) *reinterpret_cast<TreeTotals *>(ws) = totals;
            long long u0 = 0;
            int left = 0;
            TreeWalk w;
            if (cta < deal.ctas) {
                u0 = deal.first(cta);
                left = (int)(deal.first(cta + 1) - u0);
                w.begin(a, p, totals, u0, s0, c0);
                left = max(left - w.ahead, 0);
            }
            TreeItem it = {};
            auto make = [&] {
                it.stop = 1;
                if (left == 0) return;
                const int rec = w.own ? p.own_rec : p.pre_rec;
                it.own = w.own;
                it.b = w.b;
                it.kh = w.kh;
                it.rt = w.rt;
                it.tile = w.tile;
                it.count = min(w.tiles - w.tile, left);
                it.len = w.len;
                it.rows = w.rows(p);
                it.t0 = w.t0;
                it.rec = (long long)(w.item + cta) * rec;
                left -= it.count;
                it.stop = left <= totals.change;
            };
            make();
            constexpr int kBufs = TWO ? 1 : 2;
            int told = 0, brought = 0;                          // items said, items whose rows of Q are there or under way
            bool all = false;
            // It moves when an item ends, which is as long away as the longest under way takes (a unit 1.5 us, here 20).
            unsigned long long t0 = global_ns(), longest = 0;
            while (!all || brought < told) {
                bool moved = false;
                const int i = told & (kTrItems - 1), buf = brought % kBufs;
                if (!all && told < brought + kTrItems && __all_sync(0xffffffffu, mbar_test(&sh.item_empty[i], ((told / kTrItems) & 1) ^ 1))) {
                    if (lane == 0) {
                        sh.item[i] = it;
                        mbar_arrive(&sh.item_full[i]);
                    }
                    __syncwarp();
                    longest = max(longest, (unsigned long long)it.count);
                    ++told;
                    all = it.stop;
                    moved = true;
                    if (!all) {
                        w.next_item(a, p);
                        left -= totals.change;
                        make();
                    }
                }
                if (brought < told && (brought < kBufs || __all_sync(0xffffffffu, mbar_test(&sh.q_free[buf], (brought / kBufs - 1) & 1)))) {
                    const TreeItem x = sh.item[brought & (kTrItems - 1)];
                    if (x.count) tree_bring<TWO>(a, p, x, sh, qs, buf, mapQ);
                    ++brought;
                    moved = true;
                }
                if (moved) t0 = global_ns();
                else if (global_ns() - t0 > kWaitLimitNs + longest * 20000) { ok = false; break; }
                else __nanosleep(40);
            }
            // (gave up: let what is under way land, bounded, before the memory goes)
            if (!ok && p.group <= 128)
                for (int i = 0; i < kBufs; ++i) mbar_wait(&sh.q_ready[i], 0);
            tree_leave(a, p, ws, cta, totals.change);
        } else if (warp == 0) {
            // ---------------------------------------------------------- copies: a unit's keys, then its values
            TreeItems items;
            TreeItem it, next;
            ok = items.next(sh, it);
            int s = 0, tile = it.tile, left = it.count, g = 0, told = 0;    // g: the unit, told: tiles of it that are under way
            uint32_t ph = 0, unused;
            auto entry = [&](const TreeItem &x, int t, int r) {     // entry of the page list for the unit's r'th key, if there is such a key
                if (r >= x.len - t * p.unit) return 0;              // (the sum may be beyond 2^31)
                const int key = t * p.unit + r;
                return (x.own ? a.page_table + (long long)x.b * a.ld_table : a.prefix_pages)[(unsigned)key / (unsigned)a.page_size];
            };
            if (p.box) {
                const int boxes = p.unit / p.box, at = lane * p.box;
                int page = ok && left && lane < boxes ? entry(it, tile, at) : 0;
                while (ok && left > 0) {
                    const int keys = min(p.unit, it.len - tile * p.unit), kh = it.kh, row = ((unsigned)(tile * p.unit) + (unsigned)at) % (unsigned)a.page_size;
                    const bool there = lane < boxes && at < keys, bad = there && (page < 0 || page >= a.n_pages);
                    const int pid = bad ? 0 : page, n = __popc(__ballot_sync(0xffffffffu, there));
                    if (bad && (kh | it.rt | row) == 0 && a.st) atomicAdd(&a.st->out_of_range, 1ull);
                    // the next unit's page, while these stages empty
                    ++tile;
                    if (--left == 0 && !it.stop) {
                        if (!(ok = items.next(sh, next))) break;
                        it = next;
                        tile = it.tile;
                        left = it.count;
                    }
                    if (left) page = lane < boxes ? entry(it, tile, at) : 0;
#pragma unroll 1
                    for (int v = 0; v < 2; ++v) {
                        ok = __all_sync(0xffffffffu, mbar_wait(&sh.empty[s], ph ^ 1));
                        if (!ok) break;
                        uint64_t *const full = landing(g, v, &unused);
                        if (lane == 0) mbar_arrive_expect_tx(full, (uint32_t)(n * p.box * 128 * halves));
                        __syncwarp();
                        if (there)
                            for (int h = 0; h < halves; ++h)
                                tma_load4(smem_u32(tiles + s * tile_bytes + h * 16384) + at * 128, v ? &mapV : &mapK, h * 64, kh, row, pid, smem_u32(full));
                        if (++s == n_tiles) { s = 0; ph ^= 1; }
                        told = v + 1;
                    }
                    if (!ok) break;
                    ++g;
                    told = 0;
                }
            } else {
                // pages and strides that tiled copies do not serve: 16 bytes at a time, a tile's under way while the one before lands
                const int per = hd / 8;
                uint64_t *pending = nullptr;
                auto landed = [&](uint64_t *full) {
                    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                    __syncwarp();
                    if (lane == 0) mbar_arrive(full);
                    __syncwarp();
                };
                while (ok && left > 0) {
                    const int keys = min(p.unit, it.len - tile * p.unit);
                    long long off[4];                           // element of the pool of keys lane, lane + 32, ...; -1: none
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const int r = i * 32 + lane;
                        const int page = entry(it, tile, r);
                        const unsigned row = ((unsigned)(tile * p.unit) + (unsigned)r) % (unsigned)a.page_size;
                        const bool bad = r < keys && (page < 0 || page >= a.n_pages);
                        if (bad && (it.kh | it.rt) == 0 && row == 0 && a.st) atomicAdd(&a.st->out_of_range, 1ull);
                        off[i] = r < keys ? (long long)(bad ? 0 : page) * a.page_stride + (long long)row * a.token_stride + it.kh * a.head_stride : -1;
                    }
                    ++tile;
                    if (--left == 0 && !it.stop) {
                        if (!(ok = items.next(sh, next))) break;
                        it = next;
                        tile = it.tile;
                        left = it.count;
                    }
#pragma unroll 1
                    for (int v = 0; v < 2; ++v) {
                        if (pending && !__all_sync(0xffffffffu, mbar_try_wait(&sh.empty[s], ph ^ 1))) {
                            asm volatile("cp.async.wait_group 0;" ::: "memory");
                            landed(pending);
                            pending = nullptr;
                        }
                        ok = __all_sync(0xffffffffu, mbar_wait(&sh.empty[s], ph ^ 1));
                        if (!ok) break;
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
                        if (pending) {
                            asm volatile("cp.async.wait_group 1;" ::: "memory");
                            landed(pending);
                        }
                        pending = landing(g, v, &unused);
                        if (++s == n_tiles) { s = 0; ph ^= 1; }
                    }
                    if (!ok) break;
                    ++g;
                }
                asm volatile("cp.async.wait_group 0;" ::: "memory");
                if (pending) landed(pending);
            }
            if (!ok && p.box)                                   // gave up: let what is under way land (bounded) before the memory goes
                for (int t = max(2 * g + told - n_tiles, 0); t < 2 * g + told; ++t) {
                    uint32_t parity;
                    uint64_t *const full = landing(t >> 1, t & 1, &parity);
                    mbar_wait(full, parity);
                }
        } else if (!TWO || warp == 1) {
            // ---------------------------------------------------------- products: a warp for both sums of two tiles, else one for each
            const bool lead = tc_elect();
            const uint32_t idesc_s = tc_idesc_f16(D::kBf16, 128, 128, false), idesc_o = tc_idesc_f16(D::kBf16, 128, (hd + 15) / 16 * 16, true);
            const int ksteps = (hd + 15) / 16, mine = TWO ? 0 : warp - 1;
            const uint32_t q0 = tc_desc(smem_u32(qs)), kv0 = tc_desc(smem_u32(tiles)), v0 = tc_desc_mn(smem_u32(tiles), 16384);
            TreeItems items;
            TreeItem it;
            // The warp's units: all of them, or every other one.  left: those of the item, rest: keys from the next one's first on, n_item: the
            // item's number, done: all units of the items before
            constexpr int kEach = TWO ? 1 : 2;
            int left = 0, rest = 0, n_item = -1, of = 0, stop = 0, both = 0, done = 0;
            // the stages of the next K and V tiles
            int ks = 2 * mine, vs = ks + 1, kg = mine, vg = mine;           // and their units
            struct Unit { int both, fresh, steps, last, buf; };
            auto uniform = [](int x) { return __shfl_sync(0xffffffffu, x, 0); };
            auto there = [](uint64_t *bar, uint32_t parity) { return (bool)__all_sync(0xffffffffu, mbar_wait(bar, parity)); };
            // the next unit: 1, none left: 0, gave up: -1
            auto next_unit = [&](Unit &u) -> int {
                while (left == 0) {
                    if (stop) return 0;
                    if (!items.next(sh, it)) return -1;
                    const int count = uniform(it.count), first = TWO || (done & 1) == mine ? 0 : 1;
                    stop = uniform(it.stop);
                    if (count == 0) return 0;
                    left = count > first ? (count - first + kEach - 1) / kEach : 0;
                    rest = uniform(it.len - (it.tile + first) * p.unit);
                    both = TWO && uniform(it.rows) > p.part;
                    done += count;
                    of = 0;
                    ++n_item;
                    const int buf = TWO ? 0 : n_item & 1;
                    if (!there(&sh.q_ready[buf], (TWO ? n_item : n_item >> 1) & 1)) return -1;
                    if (left == 0) tc_commit<1>(&sh.q_free[buf], lead);     // (nothing of this item is this sum's)
                }
                u.both = both;
                u.fresh = of == 0;
                u.steps = (min(p.unit, rest) + 15) >> 4;
                u.last = left == 1;
                u.buf = TWO ? 0 : n_item & 1;
                rest -= kEach * p.unit;
                --left;
                ++of;
                return 1;
            };
            auto step = [&](int &stage, int &g) {
                stage += 2 * kEach;
                if (stage >= n_tiles) stage -= n_tiles;
                g += kEach;
            };
            auto tile_there = [&](int g, int v) {
                uint32_t parity;
                uint64_t *const full = landing(g, v, &parity);
                const bool r = there(full, parity);
                tc_fence_after();
                return r;
            };
            auto scores = [&](int sum, const Unit &u) {         // S = Q K^T
                const uint32_t q = q0 + (TWO ? sum : u.buf) * 2048, k = kv0 + ks * (tile_bytes >> 4);
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    if (i < ksteps) tc_mma_f16_ss(tmem + sum * 128, q + (i >> 2) * 1024 + 2 * (i & 3), k + (i >> 2) * 1024 + 2 * (i & 3), idesc_s, i > 0, lead);
                tc_commit<1>(&sh.s_full[sum], lead);
            };
            auto keys_done = [&](const Unit &u) {
                tc_commit<1>(&sh.empty[ks], lead);
                if (u.last) tc_commit<1>(&sh.q_free[u.buf], lead);
                step(ks, kg);
            };
            struct Passes { uint32_t softmax, items; } pass0 = {1, 0}, pass1 = {1, 0};
            auto values = [&](int sum, const Unit &u, Passes &n) {          // O += P V
                if (!there(&sh.p_ready[sum], n.softmax & 1)) return false;
                ++n.softmax;
                if (u.fresh) {
                    if (n.items > 0 && !there(&sh.o_free[sum], (n.items - 1) & 1)) return false;
                    ++n.items;
                }
                tc_fence_after();
                const uint32_t v = v0 + vs * (tile_bytes >> 4);
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    if (i < u.steps) tc_mma_f16_ta(tmem + 256 + sum * 128, tmem + sum * 128 + i * 8, v + i * 128, idesc_o, !u.fresh || i > 0, lead);
                tc_commit<1>(&sh.pv_done[sum], lead);
                return true;
            };
            auto values_done = [&] {
                tc_commit<1>(&sh.empty[vs], lead);
                step(vs, vg);
            };
            Unit u, next = {};
            int more = next_unit(u);
            // (the softmax's first pass writes where S will be)
            if (more > 0 && (ok = there(&sh.p_ready[mine], 0) && (!TWO || there(&sh.p_ready[1], 0)) && tile_there(kg, 0))) {
                scores(mine, u);
                if (TWO && u.both) scores(1, u);
                keys_done(u);
            }
            // each sum's scores of its next unit behind its values of this one
            while (ok && more > 0) {
                more = next_unit(next);
                if (!(ok = more >= 0 && tile_there(vg, 1) && values(mine, u, pass0))) break;
                if (!TWO) values_done();
                if (more) {
                    if (!(ok = tile_there(kg, 0))) break;
                    scores(mine, next);
                }
                if (TWO) {
                    if (u.both && !(ok = values(1, u, pass1))) break;
                    values_done();
                    if (more && next.both) scores(1, next);
                }
                if (more) keys_done(next);
                u = next;
            }
            ok = ok && more >= 0;
            // (no arrival of these products may be under way when the CTA ends)
            tc_commit<1>(&sh.issued[mine], lead);
            ok = there(&sh.issued[mine], 0) && ok;
        }
    } else {
        // -------------------------------------------------------------- softmax: two threads to a row, half of a unit's keys each
        asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kTrSoftRegs));
        const int sum = (warp - 4) >> 3, half = (warp - 4) >> 2 & 1, q4 = warp & 3, r = q4 * 32 + lane, pair = sum * 4 + q4;
        const uint32_t at = tmem + sum * 128 + ((uint32_t)(q4 * 32) << 16), acc = at + 256;
        const bool turn = a.scale < 0.0f;                       // a negative scale turns the scores' signs; a zero one must leave -inf as it is
        const float scale = (a.scale == 0.0f ? 1.17549435e-38f : fabsf(a.scale)) * 1.4426950408889634f;
        constexpr float kShift = D::kBf16 ? 0.0f : kProbabilityShift;
        // The two warps that share 32 rows wait for one another; one that gives up says so and arrives for the other.
        auto meet = [&] {
            named_bar_sync(1 + pair, 64);
            return !sh.gave_up[pair];
        };
        auto meet4 = [&] {                                      // the four that have the same rows (one tile to an item)
            named_bar_sync(9 + q4, 128);
            return !sh.gave_up[q4] && !sh.gave_up[4 + q4];
        };
        TreeItems items;
        // The first pass, on a unit that there is not, keeps nothing: it brings the code in while the first keys are under way (the
        // products wait for its P).  cnt: passes; the products of the first do not exist.
        TreeItem it = {};
        it.count = 1;
        it.len = it.rows = 256;
        bool warm = true;
        uint32_t cnt = 0;
        int done = 0;                                           // units of the items before
        do {
            if (!warm && !(ok = items.next(sh, it))) break;
            const int mine = min(it.rows - (TWO ? sum * p.part : 0), p.part);
            const bool live = q4 * 32 < mine;
            float m = -CUDART_INF_F, l = 0.0f;
            bool fresh = true;
            if (mine > 0)
                for (int u = 0; u < it.count; ++u) {
                    if (!TWO && !warm && ((done + u) & 1) != sum) continue;
                    const int keys = min(p.unit, it.len - (it.tile + u) * p.unit);
                    // values past the last key, up to the product's step of 16: zero, because a zero probability times whatever lay
                    // there (NaN, say) would not be.  (Of two tiles the first sum does it, whose product comes first; the second may have skipped
                    // items and would look at the tile's barrier phases ahead.)
                    const int zeros = (keys + 15) / 16 * 16 - keys;
                    if (zeros && (!TWO || sum == 0) && !warm) {
                        uint32_t parity;
                        uint64_t *const full = landing(done + u, 1, &parity);
                        if (!(ok = __all_sync(0xffffffffu, mbar_wait(full, parity)))) break;
                        unsigned char *const vt = tiles + (2 * (done + u) + 1) % n_tiles * tile_bytes;
                        for (int i = half * 128 + r; i < zeros * halves * 8; i += 256) {
                            const int piece = i % (halves * 8);
                            *reinterpret_cast<uint4 *>(vt + (piece >> 3) * 16384 + (keys + i / (halves * 8)) * 128 + ((piece & 7) << 4)) = make_uint4(0, 0, 0, 0);
                        }
                        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                    }
                    if (!warm && !(ok = __all_sync(0xffffffffu, mbar_wait(&sh.s_full[sum], (cnt - 1) & 1)))) break;
                    tc_fence_after();
                    if (live) {
                        uint32_t x[2][32];
                        tc_ld32(at + half * 64, x[0]);
                        tc_ld32(at + half * 64 + 32, x[1]);
                        tc_wait_ld();
                        if (turn)
#pragma unroll
                            for (int c = 0; c < 2; ++c)
#pragma unroll
                                for (int j = 0; j < 32; ++j) x[c][j] ^= 0x80000000u;
                        if (keys < half * 64 + 64)
#pragma unroll
                            for (int c = 0; c < 2; ++c)
#pragma unroll
                                for (int j = 0; j < 32; ++j)
                                    if (half * 64 + c * 32 + j >= keys) x[c][j] = 0xff800000u;
                        float top[4] = {-CUDART_INF_F, -CUDART_INF_F, -CUDART_INF_F, -CUDART_INF_F};
#pragma unroll
                        for (int c = 0; c < 2; ++c)
#pragma unroll
                            for (int j = 0; j < 32; j += 2) top[(j >> 1) & 3] = fmax3(top[(j >> 1) & 3], __uint_as_float(x[c][j]), __uint_as_float(x[c][j + 1]));
                        // the other half's maximum; past this barrier both have their scores in registers, so that P may overwrite them
                        // (and the next pass's maxima come when both have said that P is there)
                        float t = fmaxf(fmaxf(top[0], top[1]), fmaxf(top[2], top[3]));
                        sh.top[sum][half][r] = t;
                        if (!(ok = meet())) break;
                        t = fmaxf(t, sh.top[sum][half ^ 1][r]);
                        const bool above = (t - m) * scale > kTrSlack;
                        if (fresh) m = t;
                        else if (__any_sync(0xffffffffu, above && r < mine)) {
                            // a maximum well above the reference: O (half of it here) and l move to it
                            if (!(ok = __all_sync(0xffffffffu, mbar_wait(&sh.pv_done[sum], cnt & 1)))) break;       // (pass cnt - 1)
                            tc_fence_after();
                            const float to = above ? t : m, f = to == -CUDART_INF_F ? 1.0f : exp2_fast((m - to) * scale);
                            m = to;
                            l *= f;
#pragma unroll 1
                            for (int c = half * 64; c < min(hd, half * 64 + 64); c += 16) {
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
                        for (int c = 0; c < 2; ++c)
#pragma unroll
                            for (int j = 0; j < 32; j += 2) {
                                const float2 d = __ffma2_rn(__fadd2_rn(make_float2(__uint_as_float(x[c][j]), __uint_as_float(x[c][j + 1])), from2), scale2, shift2);
                                const float e = exp2_fast(d.x), f = exp2_fast(d.y);
                                part[j & 2] += e;
                                part[(j & 2) + 1] += f;
                                // rounded to the 16-bit type for the product with v; the sum takes the unrounded ones (see probability_base)
                                x[0][c * 16 + j / 2] = D::encode2(e, f);
                            }
                        tc_st32(at + half * 32, x[0]);
                        l += (part[0] + part[1]) + (part[2] + part[3]);
                        tc_wait_st();
                    }
                    tc_fence_before();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(&sh.p_ready[sum]);
                    __syncwarp();
                    ++cnt;
                    fresh = false;
                }
            if (!ok) break;
            if (warm) {
                warm = false;
                asm volatile("griddepcontrol.wait;" ::: "memory");
                continue;
            }
            done += it.count;
            if (mine <= 0 || it.count == 0) continue;
            // The CTA's record of the item.  (Eight dims of every row side by side, so that a warp's stores lie together.)
            const long long rec = it.rec + (TWO ? sum * p.part : 0) + r;        // the row's number among all records'
            float2 *const ml = reinterpret_cast<float2 *>(ws + (it.own ? p.off_own_ml : p.off_pre_ml));
            float *const dst = reinterpret_cast<float *>(ws + (it.own ? p.off_own_o : p.off_pre_o)) + tree_record(p, it.own, rec, 0, hd);
            const int step = (it.own ? p.own_rec : p.pre_rec) * 8;
            // (the shift of the probabilities is the join's to take out: behind a score of 2^24 and more it would be lost in the rounding here)
            const float base = m == -CUDART_INF_F ? m : __fmul_rn(m, scale);
            if (!fresh && !(ok = __all_sync(0xffffffffu, mbar_wait(&sh.pv_done[sum], cnt & 1)))) break;            // (pass cnt - 1)
            tc_fence_after();
            if (TWO) {
                if (live) {
                    if (half) sh.top[sum][1][r] = l;
                    if (!(ok = meet())) break;
                    if (r < mine && !half) ml[rec] = make_float2(base, l + sh.top[sum][1][r]);
                    __syncwarp();
                    if (!(ok = meet())) break;                  // (read before the next pass overwrites it)
#pragma unroll 1
                    for (int c = half * 64; c < min(hd, half * 64 + 64); c += 32) {
                        uint32_t o[32];
                        __syncwarp();
                        tc_ld32(acc + c, o);
                        tc_wait_ld();
                        if (r < mine)
#pragma unroll
                            for (int j = 0; j < 32; j += 8)
                                if (c + j < hd) {
                                    float v[8];
#pragma unroll
                                    for (int i = 0; i < 8; ++i) v[i] = __uint_as_float(o[j + i]);
                                    store32(dst + ((c + j) >> 3) * step, v);
                                }
                    }
                }
            } else if (live) {
                // The two sums of the same rows become one: the four threads of a row exchange bases and sums, each takes 32 dims of both.
                // (Of a sum that had no unit O may be anything.)
                if (half) sh.top[sum][1][r] = l;
                if (!(ok = meet())) break;
                if (!half) {
                    sh.top[sum][0][r] = fresh ? -CUDART_INF_F : base;
                    sh.top[sum][1][r] = fresh ? 0.0f : l + sh.top[sum][1][r];
                }
                tc_fence_before();
                if (!(ok = meet4())) break;
                tc_fence_after();
                const float b0 = sh.top[0][0][r], b1 = sh.top[1][0][r], l0 = sh.top[0][1][r], l1 = sh.top[1][1][r];
                const float to = fmaxf(b0, b1), from = to == -CUDART_INF_F ? 0.0f : to, f0 = exp2_fast(b0 - from), f1 = exp2_fast(b1 - from);
                const bool only0 = it.count < 2 && ((done - it.count) & 1) == 0, only1 = it.count < 2 && !only0;
                if (r < mine && sum == 0 && !half) ml[rec] = make_float2(to, only0 ? l0 : only1 ? l1 : l0 * f0 + l1 * f1);
                __syncwarp();
                if (!(ok = meet4())) break;                     // (all have read what the next pass overwrites)
                const int c = (sum * 2 + half) * 32;
                if (c < hd) {
                    uint32_t x[32], y[32];
                    tc_ld32(acc - sum * 128 + c, x);
                    tc_ld32(acc - sum * 128 + 128 + c, y);
                    tc_wait_ld();
                    if (r < mine)
#pragma unroll
                        for (int j = 0; j < 32; j += 8)
                            if (c + j < hd) {
                                float v[8];
#pragma unroll
                                for (int i = 0; i < 8; ++i) {
                                    const float p0 = __uint_as_float(x[j + i]), p1 = __uint_as_float(y[j + i]);
                                    v[i] = only0 ? p0 : only1 ? p1 : p0 * f0 + p1 * f1;
                                }
                                store32(dst + ((c + j) >> 3) * step, v);
                            }
                }
            }
            tc_fence_before();
            __syncwarp();
            if (lane == 0) {
                if (TWO) mbar_arrive(&sh.o_free[sum]);
                else {
                    // (both sums' O have been read; a sum without a unit has no products to wait)
                    if (it.count > 1 || ((done - it.count) & 1) == 0) mbar_arrive(&sh.o_free[0]);
                    if (it.count > 1 || ((done - it.count) & 1) == 1) mbar_arrive(&sh.o_free[1]);
                }
            }
            __syncwarp();
        } while (!it.stop);
        if (!ok) {
            if (lane == 0) sh.gave_up[pair] = 1;
            __syncwarp();
            named_bar_arrive(1 + pair, 64);
            if (!TWO) named_bar_arrive(9 + q4, 128);
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
// A CTA per token and run of its heads.  Which nodes the token sees and where their keys lie is looked up once; a warp takes HB heads of
// one key head at a time, for which it reads a node's key and value once, joins the nodes with the records of the units' launch, and
// writes the heads.  Its halves take turns at nodes and records, 16 lanes with eight dims each; binary32 throughout.  Bound by its
// instructions: with a warp to a single head 990 of them a row and 67 us for 1548 tokens of 32 heads; with four 51 us, 300 tokens 18 us.
constexpr int kTjWarps = 8;
template <class D, int HB>
__global__ void __launch_bounds__(kTjWarps * 32, HB == 4 ? 2 : 3)
tree_join_kernel(const TreeArgs a, const TreePlan p, int parts, const unsigned char *ws)
{
    constexpr int U = HB == 4 ? 2 : 4;                          // nodes of a half under way
    __shared__ long long place[64 * kPlanMaxWords];             // element of the pools (before the head) of each visible node
    __shared__ int counts[kTjWarps];
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, half = lane >> 4, d0 = (lane & 15) * 8, hd = a.head_dim, G = p.group;
    const int tok = (int)(blockIdx.x / (unsigned)parts), part = (int)(blockIdx.x - (unsigned)tok * (unsigned)parts), blocks = a.n_heads / HB;
    const bool in = d0 < hd;
    // (does not depend on the launch before this one)
    const unsigned long long bits = tid >> 6 < a.words ? (unsigned long long)a.mask[(long long)tok * a.words + (tid >> 6)] : 0ull;
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const TreeTotals totals = *reinterpret_cast<const TreeTotals *>(ws);
    const int b = reinterpret_cast<const int *>(ws + p.off_seq)[tok];
    if (tok >= totals.tokens || b < 0 || b >= a.n_seq) return;
    const TreeFirst s = reinterpret_cast<const TreeFirst *>(ws + sizeof(TreeTotals))[b];
    const int node = tok - s.t0;
    if (node < 0 || node >= s.nodes) return;                    // (more nodes than there may be: counted, not computed)
    // the nodes that this one sees; a thread per bit, a warp per half word (a length below the number of nodes: the first have no key)
    const int key = (int)((unsigned)s.base + (unsigned)tid);     // (looked at below 2^31 only: where the node has a place)
    const bool placed = tid < s.placed && key >= 0, sees = (bits >> (tid & 63) & 1) && placed;
    const uint32_t seen = __ballot_sync(0xffffffffu, sees);
    if (lane == 0) counts[warp] = __popc(seen);
    long long at = 0;
    if (sees || (tid == node && placed)) {
        const unsigned pg = (unsigned)key / (unsigned)a.page_size, row = (unsigned)key - pg * (unsigned)a.page_size;
        int page = a.page_table[(long long)b * a.ld_table + pg];
        const bool bad = page < 0 || page >= a.n_pages;
        // a page that is none counts where its first key is
        if (bad && tid == node && row == 0 && part == 0 && a.st) atomicAdd(&a.st->out_of_range, 1ull);
        if (bad) page = 0;
        at = (long long)page * a.page_stride + (long long)row * a.token_stride;
    }
    __syncthreads();
    int nodes = 0, before = 0;
#pragma unroll
    for (int i = 0; i < kTjWarps; ++i) {
        if (i < warp) before += counts[i];
        nodes += counts[i];
    }
    if (sees) place[before + __popc(seen & ((1u << lane) - 1))] = at;
    __syncthreads();
    const float scale = a.scale * 1.4426950408889634f;
    constexpr float kRecord = D::kBf16 ? 1.0f : 1.0f / 128.0f;  // 2^-kProbabilityShift: what a record has is as much larger
    const bool none = nodes == 0 && s.base <= 0 && a.prefix_len == 0;
    for (int block = part * kTjWarps + warp; block < blocks; block += parts * kTjWarps) {
        const int h = block * HB, kh = h / G, g = h - kh * G;
        const long long kv = kh * a.head_stride + d0;
        float q[HB][8], m[HB], l[HB], o[HB][8];
#pragma unroll
        for (int i = 0; i < HB; ++i) {
            m[i] = -CUDART_INF_F;
            l[i] = 0.0f;
            widen8<D>(in ? *reinterpret_cast<const uint4 *>(a.q + (long long)tok * a.ldq + (long long)(h + i) * hd + d0) : make_uint4(0, 0, 0, 0), q[i]);
#pragma unroll
            for (int j = 0; j < 8; ++j) o[i][j] = 0.0f;
        }
        // ---- nodes
        for (int i0 = half; i0 < nodes + half; i0 += 2 * U) {   // (both halves make the same steps)
            uint4 k[U], v[U];
            float sc[U][HB];
#pragma unroll
            for (int i = 0; i < U; ++i) {
                const int n = i0 + 2 * i;
                k[i] = v[i] = make_uint4(0, 0, 0, 0);
                if (n < nodes && in) {
                    const long long x = place[n] + kv;
                    k[i] = *reinterpret_cast<const uint4 *>(a.ck + x);
                    v[i] = *reinterpret_cast<const uint4 *>(a.cv + x);
                }
            }
#pragma unroll
            for (int i = 0; i < U; ++i) {
                float f[8];
                widen8<D>(k[i], f);
#pragma unroll
                for (int c = 0; c < HB; ++c) {
                    sc[i][c] = 0.0f;
#pragma unroll
                    for (int j = 0; j < 8; ++j) sc[i][c] = __fmaf_rn(q[c][j], f[j], sc[i][c]);
                }
            }
#pragma unroll
            for (int y = 8; y > 0; y >>= 1)
#pragma unroll
                for (int i = 0; i < U; ++i)
#pragma unroll
                    for (int c = 0; c < HB; ++c) sc[i][c] += __shfl_xor_sync(0xffffffffu, sc[i][c], y);
#pragma unroll
            for (int c = 0; c < HB; ++c) {
                float to = m[c];
#pragma unroll
                for (int i = 0; i < U; ++i) {
                    sc[i][c] = i0 + 2 * i < nodes ? sc[i][c] * scale : -CUDART_INF_F;
                    to = fmaxf(to, sc[i][c]);
                }
                const float base = to == -CUDART_INF_F ? 0.0f : to, f = exp2_fast(m[c] - base);
                m[c] = to;
                l[c] *= f;
#pragma unroll
                for (int j = 0; j < 8; ++j) o[c][j] *= f;
#pragma unroll
                for (int i = 0; i < U; ++i) {
                    // (a node that there is not has the value zero, and no part in the sum)
                    sc[i][c] = i0 + 2 * i < nodes ? exp2_fast(sc[i][c] - base) : 0.0f;
                    l[c] += sc[i][c];
                }
            }
#pragma unroll
            for (int i = 0; i < U; ++i) {
                float w[8];
                widen8<D>(v[i], w);
#pragma unroll
                for (int c = 0; c < HB; ++c)
#pragma unroll
                    for (int j = 0; j < 8; ++j) o[c][j] = __fmaf_rn(w[j], sc[i][c], o[c][j]);
            }
        }
        // ---- records: of the CTAs that had units of the key head's items, on the prefix and on the sequence's own keys.  Four lanes find
        // the first and the last CTA of the two.  (The heads' rows follow one another, in one tile: tiles hold whole tokens, or one
        // head at a time comes here.)
        const unsigned in_all = (unsigned)(tok * G + g), in_seq = (unsigned)(node * G + g), rt0 = in_all / (unsigned)p.rows, rt1 = in_seq / (unsigned)p.rows;
        const long long item0 = (long long)kh * totals.pre_rt + rt0;
        const int within = kh * s.n_rt + (int)rt1;
        const int tiles = lane & 2 ? s.tiles : p.pre_tiles;
        const long long u = (lane & 2 ? totals.pre + s.unit : 0) + ((lane & 2) ? (long long)within : item0) * (tiles + totals.change) + totals.change +
                            (lane & 1 ? tiles - 1 : 0);
        AttentionDeal deal(0, 1);
        deal.each = totals.each;
        deal.more = totals.more;
        const bool there = lane & 2 ? s.base > 0 : p.pre_tiles > 0;
        const int c = there ? deal.cta_of(u) : lane & 1 ? -1 : 0;
        const int c0 = __shfl_sync(0xffffffffu, c, 0), n0 = __shfl_sync(0xffffffffu, c, 1) - c0 + 1;
        const int c2 = __shfl_sync(0xffffffffu, c, 2), n1 = __shfl_sync(0xffffffffu, c, 3) - c2 + 1;
        const long long rec0 = item0 + c0, rec1 = (long long)(s.item + within + c2) - n0;
        const int in0 = (int)(in_all - rt0 * (unsigned)p.rows), in1 = (int)(in_seq - rt1 * (unsigned)p.rows);
        for (int k = half; k < n0 + n1; k += 2) {
            const bool own = k >= n0;
            const int n = own ? p.own_rec : p.pre_rec, row = own ? in1 : in0;
            const long long rec = (own ? rec1 : rec0) + k;
            const float2 *const ml = reinterpret_cast<const float2 *>(ws + (own ? p.off_own_ml : p.off_pre_ml)) + rec * n + row;
            const float *const src = reinterpret_cast<const float *>(ws + (own ? p.off_own_o : p.off_pre_o)) + rec * n * hd + d0 * n + row * 8;
            float2 y[HB];
            float4 v[HB][2];
#pragma unroll
            for (int i = 0; i < HB; ++i) {
                y[i] = ml[i];
                v[i][0] = in ? *reinterpret_cast<const float4 *>(src + i * 8) : make_float4(0, 0, 0, 0);
                v[i][1] = in ? *reinterpret_cast<const float4 *>(src + i * 8 + 4) : make_float4(0, 0, 0, 0);
            }
#pragma unroll
            for (int i = 0; i < HB; ++i) {
                if (y[i].x == -CUDART_INF_F && y[i].y == 0.0f) continue;        // (its output may be anything)
                const float to = fmaxf(m[i], y[i].x), f = m[i] == -CUDART_INF_F ? 0.0f : exp2_fast(m[i] - to), e = exp2_fast(y[i].x - to) * kRecord;
                l[i] = l[i] * f + y[i].y * e;                   // (a sum that is no number stays one)
                m[i] = to;
                const float w[8] = {v[i][0].x, v[i][0].y, v[i][0].z, v[i][0].w, v[i][1].x, v[i][1].y, v[i][1].z, v[i][1].w};
#pragma unroll
                for (int j = 0; j < 8; ++j) o[i][j] = o[i][j] * f + w[j] * e;
            }
        }
        // ---- the halves together
#pragma unroll
        for (int i = 0; i < HB; ++i) {
            const float m1 = __shfl_xor_sync(0xffffffffu, m[i], 16), l1 = __shfl_xor_sync(0xffffffffu, l[i], 16);
            const float to = fmaxf(m[i], m1), base = to == -CUDART_INF_F ? 0.0f : to, f = exp2_fast(m[i] - base), e = exp2_fast(m1 - base);
            const float inv = 1.0f / (l[i] * f + l1 * e), f1 = f * inv, e1 = e * inv;
#pragma unroll
            for (int j = 0; j < 8; ++j) o[i][j] = none ? 0.0f : o[i][j] * f1 + __shfl_xor_sync(0xffffffffu, o[i][j], 16) * e1;
            if (in && half == 0)
                *reinterpret_cast<uint4 *>(a.out + (long long)tok * a.ldo + (long long)(h + i) * hd + d0) =
                    make_uint4(D::encode2(o[i][0], o[i][1]), D::encode2(o[i][2], o[i][3]), D::encode2(o[i][4], o[i][5]), D::encode2(o[i][6], o[i][7]));
        }
    }
}

template <class D, int HB>
static aweq_status tree_join(const TreeArgs &a, const TreePlan &p, unsigned char *ws, cudaStream_t stream)
{
    // a token's heads over several CTAs while the tokens alone do not give every SM two
    const int most = (a.n_heads / HB + kTjWarps - 1) / kTjWarps;
    int parts = (2 * kSmCount + a.max_tokens - 1) / a.max_tokens;
    if (parts > most) parts = most;
    AWEQ_LAUNCH((tree_join_kernel<D, HB>), dim3((unsigned)a.max_tokens * (unsigned)parts), dim3(kTjWarps * 32), 0, stream, a, p, parts,
                (const unsigned char *)ws);
    return AWEQ_OK;
}

template <class D, bool TWO>
static aweq_status tree_units(const TreeArgs &a, const TreePlan &p, unsigned char *ws, cudaStream_t stream)
{
    CUtensorMap mk = {}, mv = {}, mq = {};
    aweq_status rc = AWEQ_OK;
    if (p.box) {
        rc = tma_pool_map(&mk, a.ck, a.n_pages, a.page_size, a.n_kv, a.head_dim, a.page_stride, a.token_stride, a.head_stride, p.box);
        if (rc == AWEQ_OK)
            rc = tma_pool_map(&mv, a.cv, a.n_pages, a.page_size, a.n_kv, a.head_dim, a.page_stride, a.token_stride, a.head_stride, p.box);
    }
    if (rc == AWEQ_OK && p.group <= 128) rc = tma_heads_map(&mq, a.q, a.max_tokens, a.n_heads, a.head_dim, a.ldq, p.group, p.part / p.group);
    if (rc != AWEQ_OK) return rc;
    static std::atomic<unsigned long long> allowed{0};
    AWEQ_CUDA_OK(allow_smem(tree_units_kernel<D, TWO>, kTrSmem, allowed));
    AWEQ_LAUNCH((tree_units_kernel<D, TWO>), dim3((unsigned)p.ctas), dim3(kTrThreads), kTrSmem, stream, a, p, mk, mv, mq, ws);
    return AWEQ_OK;
}

template <class D>
static aweq_status tree_launch(const TreeArgs &a, const TreePlan &p, unsigned char *ws, cudaStream_t stream)
{
    const aweq_status rc = p.two ? tree_units<D, true>(a, p, ws, stream) : tree_units<D, false>(a, p, ws, stream);
    if (rc != AWEQ_OK) return rc;
    // heads of one key head together, where their rows lie in one tile
    if (p.group <= 128 && p.group % 4 == 0) return tree_join<D, 4>(a, p, ws, stream);
    if (p.group <= 128 && p.group % 2 == 0) return tree_join<D, 2>(a, p, ws, stream);
    return tree_join<D, 1>(a, p, ws, stream);
}

aweq_status run_tree_attention(const TreeArgs &a, const aweq_kv_cache *cache, void *ws, cudaStream_t stream)
{
    const TreePlan p = tree_plan(cache, a.prefix_len, a.n_seq, a.max_tokens, a.max_nodes, a.n_heads);
    unsigned char *const w = reinterpret_cast<unsigned char *>(ws);
    return cache->dt == AWEQ_F16 ? tree_launch<F16>(a, p, w, stream) : tree_launch<BF16>(a, p, w, stream);
}

}  // namespace aweq
