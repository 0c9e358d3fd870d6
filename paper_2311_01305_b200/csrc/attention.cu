// aweq_prefix_attention: n_q tokens per sequence over a shared prefix and each sequence's own keys.
//
// All rows (token, head) that read one key head share the prefix, so the prefix is a dense product of a [rows x D]
// matrix with K and V, read once per tile of rows; the own keys are a product of the n_q * G rows of one
// sequence (G heads to a key head).  An item is a tile of rows with all its keys; a unit is a tile of 64 of them.
// The units of all items in a row are dealt out evenly to a grid that fills the device once, so a CTA streams
// through parts of one or several items without ever draining its copies, whatever the lengths are (the own ones are
// known on the device only): so many CTAs take the prefix and so many the own keys as their units ask for.  Where a CTA
// leaves an item it writes a record (base m near the maximum, sum l, output o of the keys it has seen, for each row).  A prefix with many
// rows goes to a launch of its own (attention_tc.cu), which the own keys' CTAs follow as it ends.  The last launch joins the
// records of a row:
//   m = max m_i,  l = sum 2^(m_i - m) l_i,  out = sum 2^(m_i - m) o_i / l      (scores in units of log 2)
//
// In a CTA four warps copy into a ring of stages and four compute with mma.sync, with most of the registers.  Units of the
// prefix come as tiled copies of one warp; own keys, whose pages, lengths and rows of q change from item to item, as
// 16-byte copies, 16 rows of a unit to a warp (96 sequences of 350 own keys: 43.5 us against 46 with tiled copies; 32 rows x
// 2048 shared keys and 4800 own ones: 41.9 against 45 with 16-byte copies throughout; a bulk copy per row: 40 cycles each).
// What bounds it (times on the device, replayed from a graph): memory where the keys are many (16 sequences of 1-4 thousand own keys, 32 heads of 128: 111 us, 6.05 TB/s, 94 % of
// a copy's rate), the changes from item to item where they are few (128 sequences of 64-256 keys: 78 us, 4.3 TB/s), and
// the start: the code itself comes from memory, 1 us a stretch, which is why the copying loop has one place for each step
// and the computing warps run through theirs once before the first keys are there.
#include "attention.cuh"
#include "tensorcore.cuh"

namespace aweq {

constexpr int kAtTile = 64;                 // keys of a unit
constexpr int kAtStages = 3;
constexpr int kAtThreads = 256;             // four computing warps, four that copy
// registers of a computing / copying thread: their mean is what the launch gives every thread (two CTAs of 256)
constexpr int kAtComputeRegs = 200, kAtCopyRegs = 56;

constexpr int kAtCtasPerSm = 2;

static size_t up256(size_t b) { return (b + 255) & ~(size_t)255; }

// The tensor kernel copies boxes of `box` keys that lie in one page (rows a multiple of eight, so that they keep the
// swizzle's phase) and takes as many as fit 128 keys for a unit.  Page sizes of which less than 96 keys fit are left to
// the other kernel.
static void tensor_unit(int page_size, int *unit, int *box)
{
    *unit = *box = 0;
    if (page_size % 8) return;
    if (page_size <= 128) *box = page_size;
    else if (page_size % 128 == 0) *box = 128;
    else if (page_size % 64 == 0) *box = 64;
    else return;
    *unit = 128 / *box * *box;
}

// Whether the prefix goes to the tensor kernel: more than 32 rows per key head (the other kernel's 16-row tiles serve 32
// rows at the rate of the copies: 32 rows x 8192 keys x 32 heads of 128, 47.1 us against 46.4; 96 rows, 99.9 against 69.9)
// and three units for every SM (its start is slower: 64 rows x 1024 keys x 12 heads of 64, 18.6 us against 21.0).
static bool attention_prefers_tensor(long long rows, long long units)
{
    return rows > 32 && units * ((rows + 127) / 128) >= 3 * kSmCount;
}

static AttentionPlan attention_plan(const aweq_kv_cache *c, long long prefix_len, long long max_own, long long n_seq, int n_q,
                                    int n_heads)
{
    AttentionPlan p;
    const int n_kv = c->n_kv_heads, head_dim = c->head_dim;
    const long long pre_rows = n_seq * n_q * (n_heads / n_kv), own_rows = (long long)n_q * (n_heads / n_kv);
    p.dp = head_dim <= 64 ? 64 : head_dim <= 96 ? 96 : 128;
    p.rows = n_seq * n_q * n_heads;
    tensor_unit(c->page_size, &p.pre_unit, &p.box);
    p.unit = kAtTile;
    p.tensor = p.pre_unit >= 96 && prefix_len > 0 && tma_pool_fits(c->page_stride, c->token_stride, c->head_stride) &&
               attention_prefers_tensor(pre_rows, (prefix_len + p.pre_unit - 1) / p.pre_unit * n_kv);
    if (!p.tensor) p.pre_unit = p.unit;
    p.pre_tile = p.tensor ? 128 : pre_rows <= 16 ? 16 : pre_rows <= 32 ? 32 : 64;
    p.own_tile = own_rows <= 16 ? 16 : own_rows <= 32 ? 32 : 64;
    p.pre_rt = (int)((pre_rows + p.pre_tile - 1) / p.pre_tile);
    p.own_rt = (int)((own_rows + p.own_tile - 1) / p.own_tile);
    p.pre_rec = (int)(pre_rows < p.pre_tile ? pre_rows : p.pre_tile);
    p.own_rec = (int)(own_rows < p.own_tile ? own_rows : p.own_tile);
    p.pre_tiles = (prefix_len + p.pre_unit - 1) / p.pre_unit;
    p.pre_units = p.pre_tiles * n_kv * p.pre_rt;
    const long long own_items = n_seq * n_kv * p.own_rt;
    const double most = (p.tensor ? 0.0 : (double)p.pre_units) + (double)own_items * (double)((max_own + p.unit - 1) / p.unit);
    p.ctas = kSmCount * kAtCtasPerSm;
    if (most < p.ctas) p.ctas = (int)most;
    p.tc_ctas = !p.tensor ? 0 : p.pre_units < kSmCount ? (int)p.pre_units : kSmCount;
    // an item makes a record, and one more for every CTA boundary inside it
    const size_t pre_kept = p.pre_tiles ? (size_t)((long long)n_kv * p.pre_rt + (p.tensor ? p.tc_ctas : p.ctas)) * p.pre_rec : 0;
    const size_t own_kept = (size_t)(own_items + p.ctas) * p.own_rec;
    size_t off = up256((size_t)(n_seq + 2) * 8);
    p.off_pre_o = off; off += up256(pre_kept * head_dim * 4);
    p.off_pre_ml = off; off += up256(pre_kept * 8);
    p.off_own_o = off; off += up256(own_kept * head_dim * 4);
    p.off_own_ml = off; off += up256(own_kept * 8);
    p.total = off;
    return p;
}

size_t prefix_attention_ws_bytes(const aweq_kv_cache *c, long long prefix_len, long long max_own, long long n_seq, int n_q,
                                 int n_heads)
{
    return attention_plan(c, prefix_len, max_own, n_seq, n_q, n_heads).total;
}

// ------------------------------------------------------------------ device pieces
template <class D>
__device__ __forceinline__ void mma16(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1);
template <>
__device__ __forceinline__ void mma16<F16>(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1)
{
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
template <>
__device__ __forceinline__ void mma16<BF16>(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1)
{
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void ldsm4(uint32_t (&r)[4], uint32_t at)
{
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(at) : "memory");
}
__device__ __forceinline__ void ldsm4t(uint32_t (&r)[4], uint32_t at)
{
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(at) : "memory");
}
__device__ __forceinline__ void cp_async16(uint32_t dst, const void *src, bool in)      // zeros where !in (src is not read)
{
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(in ? 16 : 0) : "memory");
}
__device__ __forceinline__ float quad_max(float v)
{
    v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, 1));
    return fmaxf(v, __shfl_xor_sync(0xffffffffu, v, 2));
}
__device__ __forceinline__ float quad_sum(float v)
{
    v += __shfl_xor_sync(0xffffffffu, v, 1);
    return v + __shfl_xor_sync(0xffffffffu, v, 2);
}

// A stage: 64 rows of K and of V in halves of 64 columns (128 bytes; one half up to a head of 64), each row's 16-byte pieces
// permuted by the row's number modulo 8, as the tiled copies leave them, so that eight rows' like pieces lie in different banks;
// then 16 rows of q with 16 bytes between them to the same end.
__host__ __device__ constexpr int at_pitch(int dp) { return dp == 64 ? 128 : 256; }
__device__ __forceinline__ uint32_t at_kv(int row, int piece) { return (uint32_t)((piece >> 3) * (kAtTile * 128) + row * 128 + ((piece ^ row) & 7) * 16); }
template <int DP>
__host__ __device__ constexpr int at_q_pitch() { return DP * 2 + 16; }
template <int DP>
__host__ __device__ constexpr int attention_stage_bytes() { return (2 * kAtTile * at_pitch(DP) + 16 * at_q_pitch<DP>() + 1023) / 1024 * 1024; }

struct AttentionState {          // of a warp's 16 rows: lanes hold rows g and g + 8
    float m[2], l[2];
};

// One tile of keys for a warp's 16 rows.  WM warps of the CTA lie along the rows, 4 / WM share the keys of the tile.
template <class D, int DP, int WM, bool OWN>
__device__ __forceinline__ void attention_tile(const AttentionArgs &a, const AttentionUnit &it, uint32_t ks, const uint32_t (&q)[DP / 16][4],
                                               const int (&own_i)[2], float scale, float (&o)[DP / 8][4], AttentionState &st, bool boxes)
{
    constexpr int KW = 4 / WM, NT = kAtTile / 8 / KW;           // warps along the keys, 8-key groups of a warp
    const int lane = threadIdx.x & 31, t = lane & 3;
    const uint32_t vs = ks + kAtTile * at_pitch(DP);
    const int key0 = (int)(threadIdx.x >> 5) / WM * (NT * 8);   // this warp's keys of the tile
    float s[NT][4] = {};
#pragma unroll
    for (int k = 0; k < DP / 16; ++k)
#pragma unroll
        for (int n = 0; n < NT; n += 2) {
            uint32_t b[4];          // keys n*8.. (k halves 0, 1), keys n*8 + 8.. (k halves 0, 1)
            ldsm4(b, ks + at_kv(key0 + n * 8 + (lane & 7) + (lane >> 4) * 8, k * 2 + ((lane >> 3) & 1)));
            mma16<D>(s[n], q[k], b[0], b[1]);
            mma16<D>(s[n + 1], q[k], b[2], b[3]);
        }
    // keys of this warp's share that a row sees: token i of a sequence leaves out the last n_q - 1 - i
    const int there = it.len - (it.tile * kAtTile + key0), first = OWN ? there - (a.n_q - 1) : there;
    const bool edge = first < NT * 8;
    if (boxes && there < NT * 8) {
        // values past the last key: zero, because a zero probability times whatever a page holds there (NaN, say) would not be
        const int from = max(there, 0);
        for (int i = lane; i < (NT * 8 - from) * (DP / 8); i += 32)
            asm volatile("st.shared.v4.u32 [%0], {%1,%1,%1,%1};" ::"r"(vs + at_kv(key0 + from + i / (DP / 8), i % (DP / 8))), "r"(0) : "memory");
        __syncwarp();
    }
    float top[2] = {st.m[0], st.m[1]};
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            s[n][e] *= scale;
            if (edge && n * 8 + 2 * t + (e & 1) >= first + (OWN ? own_i[e >> 1] : 0)) s[n][e] = -CUDART_INF_F;
            top[e >> 1] = fmaxf(top[e >> 1], s[n][e]);
        }
    float base[2], f[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        top[h] = quad_max(top[h]);
        base[h] = top[h] == -CUDART_INF_F ? 0.0f : probability_base<D>(top[h]);      // (a row that has seen no key yet)
        f[h] = exp2_fast(probability_base<D>(st.m[h]) - base[h]);
        st.m[h] = top[h];
        st.l[h] *= f[h];
    }
    // rounded to the 16-bit type for the product with v, unrounded in their sum (see probability_base)
    uint32_t p[NT / 2][4];
#pragma unroll
    for (int n = 0; n < NT; ++n) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            s[n][e] = exp2_fast(s[n][e] - base[e >> 1]);
            st.l[e >> 1] += s[n][e];
        }
        p[n / 2][(n & 1) * 2] = D::encode2(s[n][0], s[n][1]);
        p[n / 2][(n & 1) * 2 + 1] = D::encode2(s[n][2], s[n][3]);
    }
    if (__any_sync(0xffffffffu, f[0] != 1.0f || f[1] != 1.0f))   // the maxima soon stay what they are
#pragma unroll
        for (int n = 0; n < DP / 8; ++n)
#pragma unroll
            for (int e = 0; e < 4; ++e) o[n][e] *= f[e >> 1];
    // Among the last keys are some that only a sequence's later tokens see.  Zero times their values is zero unless a value is
    // infinite or NaN, which is looked for.
    bool apart = false;
    if (OWN && edge && a.n_q > 1) {
        const int from = max(first, 0), to = min(there, NT * 8);
        for (int i = lane; i < (to - from) * (DP / 8); i += 32) {
            const int r = key0 + from + i / (DP / 8);
            uint4 v;
            asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w)
                         : "r"(vs + at_kv(r, i % (DP / 8))) : "memory");
            apart |= D::any_nonfinite(v);
        }
        apart = __any_sync(0xffffffffu, apart);
    }
    if (!OWN || !apart) {
#pragma unroll
        for (int k = 0; k < NT / 2; ++k)
#pragma unroll
            for (int n = 0; n < DP / 8; n += 2) {
                uint32_t b[4];
                ldsm4t(b, vs + at_kv(key0 + k * 16 + (lane & 15), n + (lane >> 4)));
                mma16<D>(o[n], p[k], b[0], b[1]);
                mma16<D>(o[n + 1], p[k], b[2], b[3]);
            }
    } else {
        // one token's rows at a time, with the values beyond its limit replaced by zero
        const int lo = __reduce_min_sync(0xffffffffu, min(own_i[0], own_i[1])), hi = __reduce_max_sync(0xffffffffu, max(own_i[0], own_i[1]));
        for (int i = lo; i <= hi; ++i) {
#pragma unroll
            for (int k = 0; k < NT / 2; ++k)
#pragma unroll
                for (int n = 0; n < DP / 8; n += 2) {
                    uint32_t b[4];
                    ldsm4t(b, vs + at_kv(key0 + k * 16 + (lane & 15), n + (lane >> 4)));
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const int key = k * 16 + (e & 1) * 8 + 2 * t;
                        if (key >= first + i) b[e] = 0u;
                        else if (key + 1 >= first + i) b[e] &= 0xffffu;
                    }
                    float c[4] = {}, d[4] = {};
                    mma16<D>(c, p[k], b[0], b[1]);
                    mma16<D>(d, p[k], b[2], b[3]);
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        if (own_i[e >> 1] == i) {
                            o[n][e] += c[e];
                            o[n + 1][e] += d[e];
                        }
                }
        }
    }
}

struct AttentionRing {
    uint64_t full[kAtStages], landed[kAtStages], empty[kAtStages];      // (full: by the lanes' copies, landed: by boxes)
    AttentionUnit unit[kAtStages];
    float2 ml[64];
    volatile int gave_up;        // a computing warp has
};

// The copies of a CTA's units of the prefix by one warp, as boxes of `box` keys of a page (a lane each).  What a box brings
// beyond the last key is masked, and its values are zeroed, by those who compute.  Pages are looked up a unit ahead.
template <int DP>
__device__ __forceinline__ void attention_boxes(const AttentionArgs &a, const AttentionPlan &p, AttentionWalk<false> &w, int left,
                                                unsigned char *smem, AttentionRing &ring, const CUtensorMap &mapK, const CUtensorMap &mapV,
                                                int box)
{
    constexpr int STAGE = attention_stage_bytes<DP>(), HALVES = DP > 64 ? 2 : 1;
    const int lane = threadIdx.x & 31, boxes = kAtTile / box;
    // One place for each step (the first pass only looks up a page): at the start each line of code comes from memory as well.
    AttentionUnit now = {};
    int s = 0, page = 0;
    uint32_t ph = 0;
    bool ok = true;
#pragma unroll 1
    for (int step = 0; left > 0 && step <= left; ++step) {
        AttentionUnit next = w.at;
        int entry = 0;
        if (step < left) {
            entry = lane < boxes ? w.entry(a, p, lane * box) : 0;
            next.stop = step + 1 == left;
            next.leave = next.tile + 1 == w.tiles || next.stop;
            w.advance(a, p);
        }
        if (step > 0) {
            ok = mbar_wait(&ring.empty[s], ph ^ 1);
            if (!__all_sync(0xffffffffu, ok)) { ok = false; break; }
            const int keys = now.len - now.tile * kAtTile - lane * box;
            const bool has = lane < boxes && keys > 0, bad = bad_page(a, page);
            const int n = __popc(__ballot_sync(0xffffffffu, has));
            if (lane == 0) {
                ring.unit[s] = now;
                mbar_arrive_expect_tx(&ring.landed[s], (uint32_t)(n * box * 256 * HALVES));
            }
            __syncwarp();
            if (has) {
                const uint32_t dst = smem_u32(smem) + s * STAGE + lane * box * 128, bar = smem_u32(&ring.landed[s]);
                const int row = (now.tile * kAtTile + lane * box) % (unsigned)a.page_size, pid = bad ? 0 : page;
                if (bad) count_bad_page(a, now.kh, now.rt, row);
#pragma unroll
                for (int h = 0; h < HALVES; ++h) {
                    tma_load4(dst + h * (kAtTile * 128), &mapK, h * 64, now.kh, row, pid, bar);
                    tma_load4(dst + (HALVES + h) * (kAtTile * 128), &mapV, h * 64, now.kh, row, pid, bar);
                }
            }
            if (++s == kAtStages) { s = 0; ph ^= 1; }
        }
        now = next;
        page = entry;
    }
    if (!ok) {                                                  // gave up: let what is under way land (bounded) before the memory goes
        for (int i = 0; i < kAtStages; ++i) mbar_wait(&ring.landed[i], ph ^ (i >= s ? 1u : 0u));
        if (lane == 0 && a.st) atomicAdd(&a.st->wait_timeout, 1ull);
    }
}

// CTA `cta` of the `ctas` that have the prefix / the own keys.
template <class D, int DP, int WM, bool OWN>
__device__ __forceinline__ void attention_part(const AttentionArgs &a, const AttentionPlan &p, int cta, int ctas, long long total,
                                               unsigned char *ws, unsigned char *smem, AttentionRing &ring, const CUtensorMap &mapK,
                                               const CUtensorMap &mapV, int box)
{
    constexpr int PITCH = at_pitch(DP), QP = at_q_pitch<DP>(), STAGE = attention_stage_bytes<DP>(), KW = 4 / WM;
    constexpr bool kStagedQ = OWN && WM == 1;                   // short items: their rows of q come with their first unit
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int hd = a.head_dim, G = a.n_heads / a.n_kv, rec_rows = OWN ? p.own_rec : p.pre_rec;
    const bool boxes = !OWN && box;
    uint64_t *const full = boxes ? ring.landed : ring.full, *const empty = ring.empty;
    AttentionUnit *const unit = ring.unit;
    float2 *const sh_ml = ring.ml;

    if (warp >= 4) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kAtCopyRegs));
        const int cw = warp - 4;
        AttentionWalk<OWN> w;
        int left = attention_begin<OWN>(a, p, cta, ctas, total, w);
        if (left == 0) {
            if (cw == 0 && lane == 0) unit[0].stop = 2;
            mbar_arrive(&full[0]);
            if (cw == 0 && lane == 0) mbar_arrive(&full[0]);
        }
        if constexpr (!OWN)
            if (box) {
                if (cw == 0) attention_boxes<DP>(a, p, w, left, smem, ring, mapK, mapV, box);
                return;
            }
        // lanes 0-15 know this warp's 16 rows of a unit; a lane copies the same 16-byte piece of every (32 / CH)-th
        constexpr int CH = DP / 8 == 12 ? 16 : DP / 8, R = 32 / CH;
        const int mine = cw * 16 + (lane & 15), piece = lane % CH * 8;
        const uint16_t *const kp = a.ck + (piece < hd ? piece : 0), *const vp = a.cv + (piece < hd ? piece : 0);
        int page = left > 0 ? w.entry(a, p, mine) : 0;
        int s = 0;
        uint32_t ph = 0;
        bool ok = true, fresh = true;
        for (; left > 0; --left) {
            const AttentionUnit now = w.at;
            const bool leave = now.tile + 1 == w.tiles || left == 1;
            const bool has = w.has(p, mine), bad = bad_page(a, page);
            const int pg = bad ? 0 : page;
            w.advance(a, p);
            if (left > 1) page = w.entry(a, p, mine);           // the next unit's page, while this one's stage empties
            const unsigned row = (unsigned)(now.tile * kAtTile + mine) % (unsigned)a.page_size;
            if (has && bad && lane < 16) count_bad_page(a, now.kh, now.rt, row);
            // element offset of the row, -1: no such key
            const long long off = !has ? -1 : (long long)pg * a.page_stride + (long long)row * a.token_stride + now.kh * a.head_stride;
            ok = mbar_wait(&empty[s], ph ^ 1);
            if (!__all_sync(0xffffffffu, ok)) { ok = false; break; }
            if (cw == 0 && lane == 0) {
                unit[s] = now;
                unit[s].leave = leave;
                unit[s].stop = left == 1;
                mbar_arrive(&full[s]);
            }
            // missing rows become zeros, so that a zero probability times what lies there is zero
            const uint32_t dst = smem_u32(smem) + s * STAGE;
#pragma unroll
            for (int i = 0; i < 16 / R; ++i) {
                const long long o = __shfl_sync(0xffffffffu, off, i * R + lane / CH);
                const long long at = o < 0 ? 0 : o;
                const uint32_t to = dst + at_kv(cw * 16 + i * R + lane / CH, lane % CH);
                // (zeros in the columns past head_dim too: an item's sums may have lain there since)
                cp_async16(to, kp + at, o >= 0 && piece < hd);
                cp_async16(to + kAtTile * PITCH, vp + at, o >= 0 && piece < hd);
            }
            if (kStagedQ && fresh) {
                // the item's rows of q (four a warp)
                for (int r = cw * 4 + lane / CH; r < min(cw * 4 + 4, p.own_rec); r += R) {
                    const unsigned tok = now.b * a.n_q + (unsigned)r / (unsigned)G, head = now.kh * G + (unsigned)r % (unsigned)G;
                    if (piece < hd)
                        cp_async16(dst + 2 * kAtTile * PITCH + r * QP + piece * 2, a.q + (long long)tok * a.ldq + (long long)head * hd + piece, true);
                }
            }
            fresh = leave;
            asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];" ::"r"(smem_u32(&full[s])) : "memory");
            if (++s == kAtStages) { s = 0; ph ^= 1; }
        }
        if (!ok) {                                              // gave up: let what is under way land (bounded) before the memory goes
            for (int i = 0; i < kAtStages; ++i) mbar_wait(&full[i], ph ^ (i >= s ? 1u : 0u));
            if (lane == 0 && a.st) atomicAdd(&a.st->wait_timeout, 1ull);
        }
        return;
    }

    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kAtComputeRegs));
    const int g = lane >> 2, t = lane & 3, wrow = warp % WM * 16;
    uint32_t q[DP / 16][4];
    float o[DP / 8][4];
    AttentionState st;
    int own_i[2] = {0, 0}, nrows = 0;
    bool fresh = true;
    const float scale = a.scale * 1.4426950408889634f;
    int s = 0;
    uint32_t ph = 0;
    // The four warps wait for one another where they share rows; one that gives up says so and arrives for the others.
    auto meet = [&] {
        named_bar_sync(1, 128);
        return !ring.gave_up;
    };
    // The first pass computes nothing that is kept: it brings the code of the loop in, and the first rows of a prefix item's q,
    // while the first copies are under way.
    bool warm = true, q_there = false;
#pragma unroll
    for (int k = 0; k < DP / 16; ++k)
#pragma unroll
        for (int e = 0; e < 4; ++e) q[k][e] = 0u;
    AttentionUnit it = {};
    it.len = 0x40000000;
    if (!OWN) {
        const AttentionDeal deal(total, ctas);
        const int item = cta < deal.ctas ? (int)div_units(deal.first(cta), (int)p.pre_tiles) : 0;
        it.kh = item / p.pre_rt;
        it.rt = item % p.pre_rt;
    }
    for (;;) {
        if (!warm) {
            const bool ok = mbar_wait(&full[s], ph);
            if (!__all_sync(0xffffffffu, ok)) {
                if (lane == 0) {
                    if (a.st) atomicAdd(&a.st->wait_timeout, 1ull);
                    ring.gave_up = 1;
                }
                __syncwarp();
                named_bar_arrive(1, 128);
                return;
            }
            it = unit[s];
            if (it.stop == 2) return;
        }
        const uint32_t ks = smem_u32(smem + s * STAGE);
        if (fresh) {
            if (OWN ? !warm : !q_there) {
                // rows of a key head: token * G + head in group
                const int base = (OWN ? it.b * a.n_q * G : 0) + it.rt * 16 * WM;
                nrows = min((OWN ? 1 : (int)a.n_seq) * a.n_q * G - it.rt * 16 * WM, 16 * WM);
                // q as A fragments, rows g and g + 8 (rows past nrows: whatever, nobody reads what they give)
                const unsigned row_a = base + min(wrow + g, nrows - 1), row_b = base + min(wrow + g + 8, nrows - 1);
                const unsigned tok_a = row_a / (unsigned)G, tok_b = row_b / (unsigned)G;
                if (OWN) {
                    own_i[0] = (int)tok_a - it.b * a.n_q;
                    own_i[1] = (int)tok_b - it.b * a.n_q;
                }
                if (kStagedQ) {
#pragma unroll
                    for (int k = 0; k < DP / 16; ++k)
                        ldsm4(q[k], ks + 2 * kAtTile * PITCH + (lane & 15) * QP + (k * 2 + (lane >> 4)) * 16);
                } else {
                    const uint16_t *const sa = a.q + (long long)tok_a * a.ldq + (long long)(it.kh * G + (int)(row_a % (unsigned)G)) * hd + 2 * t;
                    const uint16_t *const sb = a.q + (long long)tok_b * a.ldq + (long long)(it.kh * G + (int)(row_b % (unsigned)G)) * hd + 2 * t;
#pragma unroll
                    for (int k = 0; k < DP / 16; ++k)
#pragma unroll
                        for (int e = 0; e < 2; ++e) {
                            const int d = k * 16 + e * 8;
                            q[k][2 * e] = d < hd ? *reinterpret_cast<const uint32_t *>(sa + d) : 0u;
                            q[k][2 * e + 1] = d < hd ? *reinterpret_cast<const uint32_t *>(sb + d) : 0u;
                        }
                }
            }
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                st.m[h] = -CUDART_INF_F;
                st.l[h] = 0.0f;
            }
#pragma unroll
            for (int n = 0; n < DP / 8; ++n)
#pragma unroll
                for (int e = 0; e < 4; ++e) o[n][e] = 0.0f;
        }
        fresh = it.leave;
        q_there = false;
        attention_tile<D, DP, WM, OWN>(a, it, ks, q, own_i, scale, o, st, boxes);
        if (warm) {
            warm = false;
            fresh = q_there = true;
            continue;
        }
        if (it.leave) {
            // the CTA's record of the item
            const int item = OWN ? (it.b * a.n_kv + it.kh) * p.own_rt + it.rt : it.kh * p.pre_rt + it.rt;
            const long long rec = (long long)(item + cta) * rec_rows;
            float *const ro = reinterpret_cast<float *>(ws + (OWN ? p.off_own_o : p.off_pre_o)) + rec * hd;
            float2 *const rml = reinterpret_cast<float2 *>(ws + (OWN ? p.off_own_ml : p.off_pre_ml)) + rec;
            if (KW > 1) {
                // The warps that share rows: each scales its output to their common maximum and leaves it in the stage just used
                // ([warp][16][DP]), then the sums are shared out over the threads.
                float *const ex = reinterpret_cast<float *>(smem + s * STAGE);
                const int gw = warp * 16 + g;
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    st.l[h] = quad_sum(st.l[h]);
                    if (t == 0) sh_ml[gw + 8 * h] = make_float2(probability_base<D>(st.m[h]), st.l[h]);
                }
                if (!meet()) return;                            // all have read the stage, and all (m, l) are there
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const int r = wrow + g + 8 * h;
                    if (r >= nrows) continue;
                    float2 x[KW];
                    float m = -CUDART_INF_F, l = 0.0f;
#pragma unroll
                    for (int k = 0; k < KW; ++k) {
                        x[k] = sh_ml[(k * WM + warp % WM) * 16 + g + 8 * h];
                        m = fmaxf(m, x[k].x);
                    }
                    const float base = m == -CUDART_INF_F ? 0.0f : m, mine = exp2_fast(probability_base<D>(st.m[h]) - base);
#pragma unroll
                    for (int k = 0; k < KW; ++k) l += exp2_fast(x[k].x - base) * x[k].y;
                    if (t == 0 && warp < WM) rml[r] = make_float2(m, l);
#pragma unroll
                    for (int n = 0; n < DP / 8; ++n)
                        *reinterpret_cast<float2 *>(ex + (gw + 8 * h) * DP + n * 8 + 2 * t) = make_float2(o[n][2 * h] * mine, o[n][2 * h + 1] * mine);
                }
                if (!meet()) return;
                for (int i = tid; i < nrows * (DP / 4); i += 128) {
                    const int r = i / (DP / 4), c = i % (DP / 4) * 4;
                    float4 v = make_float4(0, 0, 0, 0);
#pragma unroll
                    for (int k = 0; k < KW; ++k) {
                        const float4 y = *reinterpret_cast<const float4 *>(ex + (k * WM * 16 + r) * DP + c);
                        v.x += y.x; v.y += y.y; v.z += y.z; v.w += y.w;
                    }
                    if (c < hd) *reinterpret_cast<float4 *>(ro + (long long)r * hd + c) = v;
                }
            } else {
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    st.l[h] = quad_sum(st.l[h]);
                    const int r = wrow + g + 8 * h;
                    if (r >= nrows) continue;
                    float *const dst = ro + (long long)r * hd + 2 * t;
#pragma unroll
                    for (int n = 0; n < DP / 8; ++n)
                        if (n * 8 < hd) *reinterpret_cast<float2 *>(dst + n * 8) = make_float2(o[n][2 * h], o[n][2 * h + 1]);
                    if (t == 0) rml[r] = make_float2(probability_base<D>(st.m[h]), st.l[h]);
                }
            }
        }
        if (boxes && it.leave) asm volatile("fence.proxy.async.shared::cta;" ::: "memory");      // what was written here, before the next copies
        __syncwarp();
        if (lane == 0) mbar_arrive(&empty[s]);
        if (++s == kAtStages) { s = 0; ph ^= 1; }
        if (it.stop) return;
    }
}

// `chained`: behind the prefix's tensor kernel.  This one then starts without waiting for it, and ends after it for the
// join's sake.
template <class D, int DP, int WMP, int WMO>
__global__ void __launch_bounds__(kAtThreads, kAtCtasPerSm)
attention_units_kernel(const AttentionArgs a, const AttentionPlan p, const __grid_constant__ CUtensorMap mapK,
                       const __grid_constant__ CUtensorMap mapV, unsigned char *ws, int box, bool chained)
{
    extern __shared__ unsigned char raw[];
    unsigned char *const smem = reinterpret_cast<unsigned char *>((reinterpret_cast<uintptr_t>(raw) + 1023) & ~(uintptr_t)1023);
    __shared__ AttentionRing ring;
    const int tid = threadIdx.x, cta = blockIdx.x;
    if (tid == 0) {
        for (int s = 0; s < kAtStages; ++s) {
            mbar_init(&ring.full[s], 129);                      // every copying lane, and the unit itself
            mbar_init(&ring.landed[s], 1);
            mbar_init(&ring.empty[s], 4);
        }
        ring.gave_up = 0;
        mbar_init_fence();
        if (box) {
            tma_prefetch_map(&mapK);
            tma_prefetch_map(&mapV);
        }
    }
    if (a.head_dim < DP) {                                      // columns of q past head_dim: no copy writes them
        const int pieces = (DP - a.head_dim) / 8;
        for (int i = tid; i < kAtStages * 16 * pieces; i += kAtThreads)
            *reinterpret_cast<uint4 *>(smem + i / pieces / 16 * attention_stage_bytes<DP>() + 2 * kAtTile * at_pitch(DP) +
                                       i / pieces % 16 * at_q_pitch<DP>() + a.head_dim * 2 + i % pieces * 16) = make_uint4(0, 0, 0, 0);
    }
    __syncthreads();
    if (!chained) {
        asm volatile("griddepcontrol.wait;" ::: "memory");
        asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    }
    // CTAs for the prefix, by the time its units take (units of 16, 32 and 64 rows: as 4 to 5 to 8) and the changes from own
    // item to own item (as much as a unit each: 16 x 8192 shared keys and 512 items of one unit, 43 us without them, 37 with)
    const bool lead = cta == 0 && tid < 32;
    long long *const start = reinterpret_cast<long long *>(ws);
    const long long own = own_units(a, p, lead, start), pre = p.tensor ? 0 : p.pre_units;
    const float pre_cost = (float)pre * (WMP == 1 ? 4 : WMP == 2 ? 5 : 8);
    const float own_cost = ((float)own + fminf((float)own, (float)a.n_seq * (float)(a.n_kv * p.own_rt))) * (WMO == 1 ? 4 : WMO == 2 ? 5 : 8);
    int split = pre == 0 ? 0 : own == 0 ? p.ctas : min(max((int)(p.ctas * (pre_cost / (pre_cost + own_cost)) + 0.5f), 1), p.ctas - 1);
    if (split > pre) split = (int)pre;
    if (lead && tid == 0) {
        start[a.n_seq] = own;
        start[a.n_seq + 1] = split;
    }
    if (cta < split) attention_part<D, DP, WMP, false>(a, p, cta, split, pre, ws, smem, ring, mapK, mapV, box);
    else attention_part<D, DP, WMO, true>(a, p, cta - split, p.ctas - split, own, ws, smem, ring, mapK, mapV, box);
    if (chained && cta == 0) asm volatile("griddepcontrol.wait;" ::: "memory");
}

// WARPS warps per row (token, head), each with eight records' outputs under way.  A row has a handful of records in the usual
// case and some hundreds when one key head's keys are spread over the whole device; then there are few rows.  Bound by latency: lengths and
// cut, then (m, l) and the outputs, which fly together (1024 rows 5-6 us; 8 by itself, its start included, which nothing hides).
template <class D, int WARPS>
__global__ void __launch_bounds__(128)
attention_join_kernel(const AttentionArgs a, const AttentionPlan p, const unsigned char *ws)
{
    __shared__ float part[4][128], part_l[4];
    pdl_begin();
    const int lane = threadIdx.x & 31, warp = (int)(threadIdx.x >> 5) % WARPS, G = a.n_heads / a.n_kv, hd = a.head_dim;
    const unsigned r = blockIdx.x * (4 / WARPS) + (threadIdx.x >> 5) / WARPS;
    if (WARPS == 1 && r >= p.rows) return;
    const unsigned tok = r / (unsigned)a.n_heads, h = r % (unsigned)a.n_heads, kh = h / (unsigned)G, b = tok / (unsigned)a.n_q;
    const long long *start = reinterpret_cast<const long long *>(ws);
    long long total = 0, own0 = 0, own1 = 0;
    int split = p.tc_ctas;
    if (p.ctas) {
        total = start[a.n_seq];
        own0 = start[b];
        own1 = b + 1 < a.n_seq ? start[b + 1] : total;
        if (!p.tensor) split = (int)start[a.n_seq + 1];
    }
    const AttentionDeal deal(total, p.tensor ? p.ctas : p.ctas - split), pre_deal(p.pre_units, split);
    const int tiles = (int)div_units(own1 - own0, a.n_kv * p.own_rt);
    // the rows of this one's records: the prefix item's, then the own item's
    long long pre0 = 0, rec0 = 0;
    int n_pre = 0, n_all = 0;
    const int pre_step = p.pre_rec, own_step = p.own_rec;
    if (p.pre_tiles) {
        const unsigned row = tok * G + h % (unsigned)G, in = row % (unsigned)p.pre_tile;
        const long long item = (long long)kh * p.pre_rt + row / (unsigned)p.pre_tile;
        const int c0 = pre_deal.cta_of(item * p.pre_tiles);
        n_pre = pre_deal.cta_of((item + 1) * p.pre_tiles - 1) - c0 + 1;
        pre0 = (item + c0) * pre_step + in;
    }
    n_all = n_pre;
    if (tiles) {
        const unsigned row = tok % (unsigned)a.n_q * G + h % (unsigned)G, step = p.own_tile;
        const int within = kh * p.own_rt + row / step;
        const long long u = own0 + (long long)within * tiles;
        const int c0 = deal.cta_of(u);
        n_all += deal.cta_of(u + tiles - 1) - c0 + 1;
        rec0 = ((long long)b * a.n_kv * p.own_rt + within + c0) * own_step + row % step;
    }
    const float *const pre_o = reinterpret_cast<const float *>(ws + p.off_pre_o), *const own_o = reinterpret_cast<const float *>(ws + p.off_own_o);
    const float2 *const pre_ml = reinterpret_cast<const float2 *>(ws + p.off_pre_ml), *const own_ml = reinterpret_cast<const float2 *>(ws + p.off_own_ml);
    auto ml = [&](int i) { return i < n_pre ? pre_ml[pre0 + (long long)i * pre_step] : own_ml[rec0 + (long long)(i - n_pre) * own_step]; };
    constexpr int U = 8;
    const bool in = lane * 4 < hd;
    float4 v[U];
    auto fetch = [&](int i0) {
#pragma unroll
        for (int j = 0; j < U; ++j) {
            const int i = i0 + j;
            const float *src = i < n_pre ? pre_o + (pre0 + (long long)i * pre_step) * hd : own_o + (rec0 + (long long)(i - n_pre) * own_step) * hd;
            v[j] = in && i < n_all ? *reinterpret_cast<const float4 *>(src + lane * 4) : make_float4(0, 0, 0, 0);
        }
    };
    fetch(warp * U);                                            // under way while the maximum is found
    float m = -CUDART_INF_F;
    for (int i = lane; i < n_all; i += 32) m = fmaxf(m, ml(i).x);
    for (int x = 16; x > 0; x >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, x));
    const float base = m == -CUDART_INF_F ? 0.0f : m;
    float l = 0.0f;
    float4 o = make_float4(0, 0, 0, 0);
    for (int i0 = warp * U; i0 < n_all; i0 += WARPS * U) {
        if (i0 != warp * U) fetch(i0);
        float w = 0.0f, wl = 0.0f;
        if (lane < U && i0 + lane < n_all) {
            const float2 x = ml(i0 + lane);
            w = exp2_fast(x.x - base);
            wl = w * x.y;
        }
#pragma unroll
        for (int j = 0; j < U; ++j) {
            const float f = __shfl_sync(0xffffffffu, w, j);
            l += __shfl_sync(0xffffffffu, wl, j);
            if (i0 + j < n_all) { o.x += f * v[j].x; o.y += f * v[j].y; o.z += f * v[j].z; o.w += f * v[j].w; }
        }
    }
    if (WARPS > 1) {
        if (in) *reinterpret_cast<float4 *>(&part[warp][lane * 4]) = o;
        if (lane == 0) part_l[warp] = l;
        __syncthreads();
        if (warp) return;
        l = 0.0f;
        o = make_float4(0, 0, 0, 0);
#pragma unroll
        for (int k = 0; k < WARPS; ++k) {
            l += part_l[k];
            if (in) {
                const float4 x = *reinterpret_cast<const float4 *>(&part[k][lane * 4]);
                o.x += x.x; o.y += x.y; o.z += x.z; o.w += x.w;
            }
        }
    }
    if (in) {
        // no key at all: zeros (keys whose scores are all minus infinity: 0 / 0, as the softmax of them is)
        const bool none = l == 0.0f && a.prefix_len == 0 && clamp_length(a, a.own_len[b], false) < a.n_q - (int)(tok % (unsigned)a.n_q);
        const float inv = none ? 0.0f : 1.0f / l;
        *reinterpret_cast<uint2 *>(a.out + (long long)tok * a.ldo + (long long)h * hd + lane * 4) =
            make_uint2(D::encode2(o.x * inv, o.y * inv), D::encode2(o.z * inv, o.w * inv));
    }
    // without own keys no other kernel looks at the lengths
    if (!p.ctas && blockIdx.x == 0 && threadIdx.x < 32)
        for (int i = lane; i < (int)a.n_seq; i += 32) clamp_length(a, a.own_len[i], true);
}

// Keys of a tiled copy: a box lies in one page, on a row of the stage that keeps the swizzle's phase (a multiple of eight).
// 0: the four warps' 16-byte copies, for other page sizes and strides, and where the units do not even fill the device once.
static int units_box(const AttentionArgs &a, const AttentionPlan &p)
{
    if (p.tensor || !p.pre_tiles || a.page_size % 8 || p.ctas < kSmCount * kAtCtasPerSm) return 0;
    if (!tma_pool_fits(a.page_stride, a.token_stride, a.head_stride)) return 0;
    int box = 8;
    while (box < kAtTile && a.page_size % (2 * box) == 0) box *= 2;
    return box;
}

template <class D, int DP, int WMP, int WMO>
static aweq_status units_launch(const AttentionArgs &a, const AttentionPlan &p, unsigned char *ws, cudaStream_t stream)
{
    constexpr int smem = kAtStages * attention_stage_bytes<DP>() + 1024;
    CUtensorMap mk = {}, mv = {};
    const int box = units_box(a, p);
    if (box) {
        aweq_status rc = tma_pool_map(&mk, a.ck, a.n_pages, a.page_size, a.n_kv, a.head_dim, a.page_stride, a.token_stride, a.head_stride, box);
        if (rc == AWEQ_OK)
            rc = tma_pool_map(&mv, a.cv, a.n_pages, a.page_size, a.n_kv, a.head_dim, a.page_stride, a.token_stride, a.head_stride, box);
        if (rc != AWEQ_OK) return rc;
    }
    static std::atomic<unsigned long long> allowed{0};
    AWEQ_CUDA_OK(allow_smem(attention_units_kernel<D, DP, WMP, WMO>, smem, allowed));
    AWEQ_LAUNCH((attention_units_kernel<D, DP, WMP, WMO>), dim3((unsigned)p.ctas), dim3(kAtThreads), smem, stream, a, p, mk, mv, ws, box, p.tensor != 0);
    return AWEQ_OK;
}

template <class D, int DP>
static aweq_status units_dispatch(const AttentionArgs &a, const AttentionPlan &p, unsigned char *ws, cudaStream_t stream)
{
    // without a prefix here its side is what the own keys have; a prefix has at least the rows of a sequence
    const int wmo = p.own_tile / 16, wmp = p.tensor || !p.pre_tiles ? wmo : p.pre_tile / 16;
    if (wmo == 1) {
        if (wmp == 1) return units_launch<D, DP, 1, 1>(a, p, ws, stream);
        return wmp == 2 ? units_launch<D, DP, 2, 1>(a, p, ws, stream) : units_launch<D, DP, 4, 1>(a, p, ws, stream);
    }
    if (wmo == 2) return wmp == 2 ? units_launch<D, DP, 2, 2>(a, p, ws, stream) : units_launch<D, DP, 4, 2>(a, p, ws, stream);
    return units_launch<D, DP, 4, 4>(a, p, ws, stream);
}

template <class D>
static aweq_status attention_launch(const AttentionArgs &a, const AttentionPlan &p, aweq_dtype dt, unsigned char *ws, cudaStream_t stream)
{
    aweq_status rc = p.tensor ? run_attention_tc(a, p, dt, ws, stream) : AWEQ_OK;
    if (rc == AWEQ_OK && p.ctas)
        rc = p.dp == 64 ? units_dispatch<D, 64>(a, p, ws, stream) : p.dp == 96 ? units_dispatch<D, 96>(a, p, ws, stream) : units_dispatch<D, 128>(a, p, ws, stream);
    if (rc != AWEQ_OK) return rc;
    if (p.rows >= 4 * kSmCount)
        AWEQ_LAUNCH((attention_join_kernel<D, 1>), dim3((unsigned)((p.rows + 3) / 4)), dim3(128), 0, stream, a, p, (const unsigned char *)ws);
    else
        AWEQ_LAUNCH((attention_join_kernel<D, 4>), dim3((unsigned)p.rows), dim3(128), 0, stream, a, p, (const unsigned char *)ws);
    return AWEQ_OK;
}

aweq_status run_prefix_attention(const AttentionArgs &a, const aweq_kv_cache *cache, void *ws, cudaStream_t stream)
{
    const AttentionPlan p = attention_plan(cache, a.prefix_len, a.max_own, a.n_seq, a.n_q, a.n_heads);
    unsigned char *const w = reinterpret_cast<unsigned char *>(ws);
    return cache->dt == AWEQ_F16 ? attention_launch<F16>(a, p, cache->dt, w, stream) : attention_launch<BF16>(a, p, cache->dt, w, stream);
}

}  // namespace aweq
