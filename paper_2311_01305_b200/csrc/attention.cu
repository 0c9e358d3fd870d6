// aweq_prefix_attention: n_q tokens per sequence over a shared prefix and each sequence's own keys.
//
// All rows (token, head) that read one key head share the prefix, so the prefix is a dense product of a [rows x D]
// matrix with K and V, read once per tile of rows; the own keys are a product of the n_q * G rows of one
// sequence (G heads to a key head).  Both are cut along the keys into items, all items of both kinds run in
// one launch, each leaving (maximum, sum, output) of its keys for its rows, and a second launch joins them:
//   m = max m_i,  l = sum 2^(m_i - m) l_i,  out = sum 2^(m_i - m) o_i / l      (scores in units of log 2)
#include <math_constants.h>

#include "common.cuh"
#include "kernels.h"

namespace aweq {

constexpr int kAtTile = 64;                 // keys of a tile
constexpr int kAtStages = 3;
constexpr int kAtThreads = 128;
constexpr int kAtMostPrefix = 64, kAtMostOwn = 16;      // splits of the prefix, of a sequence's own keys

// How the work is cut (host; also sizes the scratch).
struct AttentionPlan {
    int dp;                      // head_dim padded to 64, 96 or 128
    int pre_wm, own_wm;          // warps along the rows of a prefix / own item (4 / wm along the keys)
    int pre_rt, own_rt;          // row tiles per key head / per sequence and key head
    int pre_splits, own_splits;  // most items along the keys
    int own_chunk;               // own keys (in tiles) that make another split worth while
    long long pre_items, own_items, rows;
    size_t off_ml, total;
};

static int rows_warps(long long rows) { return rows <= 16 ? 1 : rows <= 32 ? 2 : 4; }

static AttentionPlan attention_plan(long long prefix_len, long long max_own, long long n_seq, int n_q, int n_heads, int n_kv,
                                    int head_dim)
{
    AttentionPlan p;
    p.dp = head_dim <= 64 ? 64 : head_dim <= 96 ? 96 : 128;
    p.rows = n_seq * n_q * n_heads;
    const long long pre_rows = n_seq * n_q * (n_heads / n_kv), own_rows = (long long)n_q * (n_heads / n_kv);
    p.pre_wm = rows_warps(pre_rows);
    p.own_wm = rows_warps(own_rows);
    p.pre_rt = (int)((pre_rows + 16 * p.pre_wm - 1) / (16 * p.pre_wm));
    p.own_rt = (int)((own_rows + 16 * p.own_wm - 1) / (16 * p.own_wm));
    const long long pre_tiles = (prefix_len + kAtTile - 1) / kAtTile;
    const long long own_tiles = (max_own + kAtTile - 1) / kAtTile;
    // the chunk length (in tiles) whose items fill the SMs best: waves of two CTAs per SM, each costing its keys
    // and about three tiles of filling, draining and joining
    const long long slots = 2 * kSmCount, pre_base = (long long)n_kv * p.pre_rt, own_base = n_seq * n_kv * p.own_rt;
    double best = 0;
    p.pre_splits = p.own_splits = 0;
    p.own_chunk = 1;
    for (int t = 1; t <= 1024; t += t < 16 ? 1 : t < 128 ? 4 : 64) {
        long long ps = (pre_tiles + t - 1) / t, os = (own_tiles + t - 1) / t;
        if (ps > kAtMostPrefix) ps = kAtMostPrefix;
        if (os > kAtMostOwn) os = kAtMostOwn;
        const long long items = pre_base * ps + own_base * os;
        const long long longest = ps ? (pre_tiles + ps - 1) / ps : 0;
        const double cost = (double)((items + slots - 1) / slots) * ((longest > t ? longest : t) + 3.0);
        if (p.pre_splits + p.own_splits == 0 || cost < best) {
            best = cost;
            p.pre_splits = (int)ps;
            p.own_splits = (int)os;
            p.own_chunk = t;
        }
    }
    p.pre_items = pre_base * p.pre_splits;
    p.own_items = own_base * p.own_splits;
    const size_t slices = (size_t)(p.pre_splits + p.own_splits) * (size_t)p.rows;
    p.off_ml = (slices * head_dim * 4 + 255) & ~(size_t)255;
    p.total = p.off_ml + slices * 8 + 256;
    return p;
}

size_t prefix_attention_ws_bytes(const aweq_kv_cache *c, long long prefix_len, long long max_own, long long n_seq, int n_q,
                                 int n_heads)
{
    return attention_plan(prefix_len, max_own, n_seq, n_q, n_heads, c->n_kv_heads, c->head_dim).total;
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
__device__ __forceinline__ void cp_async_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void cp_async_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }
__device__ __forceinline__ float exp2_fast(float x)
{
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
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

// A clamped own length; every thread of every item computes the same.  `count`: the one caller that reports it.
__device__ __forceinline__ long long own_length(const AttentionArgs &a, long long b, bool count)
{
    long long len = __ldg(a.own_len + b);
    const long long most = min(a.max_own, a.pages_per_seq * a.page_size);
    if (len < 0 || len > most) {
        if (count && a.st) atomicAdd(&a.st->out_of_range, 1ull);
        len = len < 0 ? 0 : most;
    }
    return len;
}
// own items along the keys of a sequence of `tiles` tiles
__device__ __forceinline__ int own_splits_of(long long tiles, int most, int chunk)
{
    const long long n = (tiles + chunk - 1) / chunk;
    return (int)(n < most ? n : most);
}

struct AttentionItem {
    const int *pages;
    long long k0, k1;            // keys [k0, k1)
    long long limit0;            // own keys: token i of the sequence sees keys below limit0 + i; prefix: all
    long long row0;              // first row (token * G + head in group) of this key head
    int nrows, kh, slot;         // rows, key head, slice of the scratch
    bool own;
};

template <class D, int DP, int WM>
__device__ __forceinline__ void attention_item(const AttentionArgs &a, const AttentionItem &it, float *o_part, float2 *ml_part,
                                               long long rows_total, unsigned char *smem)
{
    constexpr int KW = 4 / WM, NT = kAtTile / 8 / KW;           // warps along the keys, 8-key groups of a warp
    constexpr int PITCH = DP * 2 + 16;                          // bytes of a staged row: 16 more against bank conflicts
    constexpr int STAGE = 2 * kAtTile * PITCH;
    constexpr int CH = DP / 8;                                  // 16-byte pieces of a row
    long long *const offs = reinterpret_cast<long long *>(smem + kAtStages * STAGE);          // [kAtStages + 1][kAtTile]
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, g = lane >> 2, t = lane & 3;
    const int wm = warp % WM, wk = warp / WM;
    const int G = a.n_heads / a.n_kv, hd = a.head_dim;
    const int tiles = (int)((it.k1 - it.k0 + kAtTile - 1) / kAtTile);

    // element offsets of a tile's keys (before the head), -1 past the end
    auto find = [&](int tile) {
        if (tile < tiles && tid < kAtTile) {
            const long long c = it.k0 + (long long)tile * kAtTile + tid;
            long long off = -1;
            if (c < it.k1) {
                long long page = __ldg(it.pages + (unsigned)c / (unsigned)a.page_size);
                if (page < 0 || page >= a.n_pages) {
                    if (a.st) atomicAdd(&a.st->out_of_range, 1ull);
                    page = 0;
                }
                off = page * a.page_stride + (long long)((unsigned)c % (unsigned)a.page_size) * a.token_stride + it.kh * a.head_stride;
            }
            offs[(tile % (kAtStages + 1)) * kAtTile + tid] = off;
        }
    };
    auto load = [&](int tile) {
        if (tile < tiles) {
            const uint32_t dst = smem_u32(smem + (tile % kAtStages) * STAGE);
            const long long *of = offs + (tile % (kAtStages + 1)) * kAtTile;
#pragma unroll
            for (int i = 0; i < kAtTile * CH / kAtThreads; ++i) {
                const int idx = tid + i * kAtThreads, r = idx / CH, c = idx % CH;
                const long long off = of[r];
                const bool in = off >= 0 && c * 8 < hd;
                const long long src = in ? off + c * 8 : 0;
                cp_async16(dst + r * PITCH + c * 16, a.ck + src, in);
                cp_async16(dst + (kAtTile + r) * PITCH + c * 16, a.cv + src, in);
            }
        }
        cp_async_commit();
    };
    for (int i = 0; i < kAtStages; ++i) find(i);
    __syncthreads();
    for (int i = 0; i < kAtStages - 1; ++i) load(i);

    // this warp's 16 rows of q, as A fragments: rows g and g + 8
    uint32_t q[DP / 16][4];
    long long tok[2];
    int rloc[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        rloc[h] = wm * 16 + g + h * 8;
        const long long r = it.row0 + min(rloc[h], it.nrows - 1);
        tok[h] = r / G;
        const uint16_t *src = a.q + tok[h] * a.ldq + (long long)(it.kh * G + (int)(r % G)) * hd;
#pragma unroll
        for (int k = 0; k < DP / 16; ++k)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const int d = k * 16 + e * 8 + 2 * t;
                q[k][h + 2 * e] = d < hd && rloc[h] < it.nrows ? *reinterpret_cast<const uint32_t *>(src + d) : 0u;
            }
    }
    // keys that rows g and g + 8 see
    long long lim[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) lim[h] = it.own ? it.limit0 + tok[h] % a.n_q : it.k1;
    const long long lim_min = it.own ? it.limit0 : it.k1;       // a tile below it needs no comparison

    float o[DP / 8][4] = {}, m[2] = {-CUDART_INF_F, -CUDART_INF_F}, l[2] = {0.0f, 0.0f};
    const float scale = a.scale * 1.4426950408889634f;
    for (int tile = 0; tile < tiles; ++tile) {
        cp_async_wait<kAtStages - 2>();
        __syncthreads();
        load(tile + kAtStages - 1);
        find(tile + kAtStages);
        const uint32_t ks = smem_u32(smem + (tile % kAtStages) * STAGE), vs = ks + kAtTile * PITCH;
        const int key0 = wk * (NT * 8);                          // this warp's keys of the tile
        float s[NT][4] = {};
#pragma unroll
        for (int k = 0; k < DP / 16; ++k)
#pragma unroll
            for (int n = 0; n < NT; n += 2) {
                uint32_t b[4];          // keys n*8.. (k halves 0, 1), keys n*8 + 8.. (k halves 0, 1)
                ldsm4(b, ks + (key0 + n * 8 + (lane & 7) + (lane >> 4) * 8) * PITCH + k * 32 + ((lane >> 3) & 1) * 16);
                mma16<D>(s[n], q[k], b[0], b[1]);
                mma16<D>(s[n + 1], q[k], b[2], b[3]);
            }
        const long long c0 = it.k0 + (long long)tile * kAtTile + key0;
        const bool edge = c0 + NT * 8 > lim_min;
        float top[2] = {m[0], m[1]};
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                s[n][e] *= scale;
                if (edge && c0 + n * 8 + 2 * t + (e & 1) >= lim[e >> 1]) s[n][e] = -CUDART_INF_F;
                top[e >> 1] = fmaxf(top[e >> 1], s[n][e]);
            }
        float base[2], f[2];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            top[h] = quad_max(top[h]);
            base[h] = top[h] == -CUDART_INF_F ? 0.0f : top[h];  // a row that has seen no key yet
            f[h] = exp2_fast(m[h] - base[h]);
            m[h] = top[h];
            l[h] *= f[h];
        }
        uint32_t p[NT / 2][4];          // probabilities as A fragments, rounded to the 16-bit type
#pragma unroll
        for (int n = 0; n < NT; ++n) {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                s[n][e] = exp2_fast(s[n][e] - base[e >> 1]);
                l[e >> 1] += s[n][e];
            }
            p[n / 2][(n & 1) * 2] = D::encode2(s[n][0], s[n][1]);
            p[n / 2][(n & 1) * 2 + 1] = D::encode2(s[n][2], s[n][3]);
        }
#pragma unroll
        for (int n = 0; n < DP / 8; ++n)
#pragma unroll
            for (int e = 0; e < 4; ++e) o[n][e] *= f[e >> 1];
        if (!(it.own && edge && a.n_q > 1)) {
#pragma unroll
            for (int k = 0; k < NT / 2; ++k)
#pragma unroll
                for (int n = 0; n < DP / 8; n += 2) {
                    uint32_t b[4];
                    ldsm4t(b, vs + (key0 + k * 16 + (lane & 15)) * PITCH + n * 16 + (lane >> 4) * 16);
                    mma16<D>(o[n], p[k], b[0], b[1]);
                    mma16<D>(o[n + 1], p[k], b[2], b[3]);
                }
        } else {
            // The last keys: a key may be one that only the later tokens see, and 0 * Inf of its value must not reach the
            // earlier ones.  One token's rows at a time, with the values beyond its limit replaced by zero.
            long long i0 = tok[0] % a.n_q, i1 = tok[1] % a.n_q;
            long long lo = min(i0, i1), hi = max(i0, i1);
            for (int x = 16; x > 0; x >>= 1) {
                lo = min(lo, __shfl_xor_sync(0xffffffffu, lo, x));
                hi = max(hi, __shfl_xor_sync(0xffffffffu, hi, x));
            }
            for (long long i = lo; i <= hi; ++i) {
                const long long left = it.limit0 + i - c0;       // keys of this warp's share that token i sees
#pragma unroll
                for (int k = 0; k < NT / 2; ++k)
#pragma unroll
                    for (int n = 0; n < DP / 8; n += 2) {
                        uint32_t b[4];
                        ldsm4t(b, vs + (key0 + k * 16 + (lane & 15)) * PITCH + n * 16 + (lane >> 4) * 16);
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            const long long key = k * 16 + (e & 1) * 8 + 2 * t;
                            if (key >= left) b[e] = 0u;
                            else if (key + 1 >= left) b[e] &= 0xffffu;
                        }
                        float c[4] = {}, d[4] = {};
                        mma16<D>(c, p[k], b[0], b[1]);
                        mma16<D>(d, p[k], b[2], b[3]);
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            if ((e >> 1 ? i1 : i0) == i) {
                                o[n][e] += c[e];
                                o[n + 1][e] += d[e];
                            }
                    }
            }
        }
    }
    cp_async_wait<0>();
#pragma unroll
    for (int h = 0; h < 2; ++h) l[h] = quad_sum(l[h]);

    if (KW > 1) {
        // join the warps that shared the rows: maxima and factors first, then the outputs through shared memory
        __syncthreads();
        float *const ex = reinterpret_cast<float *>(smem);       // [4 warps][16 rows] x {m, l}, then outputs
        float *const eo = ex + 4 * 16 * 2;
        if (t == 0)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                ex[(warp * 16 + g + h * 8) * 2] = m[h];
                ex[(warp * 16 + g + h * 8) * 2 + 1] = l[h];
            }
        __syncthreads();
        float all_m[2], all_l[2], mine[2];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            all_m[h] = -CUDART_INF_F;
#pragma unroll
            for (int k = 0; k < KW; ++k) all_m[h] = fmaxf(all_m[h], ex[((k * WM + wm) * 16 + g + h * 8) * 2]);
            const float b = all_m[h] == -CUDART_INF_F ? 0.0f : all_m[h];
            all_l[h] = 0.0f;
#pragma unroll
            for (int k = 0; k < KW; ++k) {
                const float *x = ex + ((k * WM + wm) * 16 + g + h * 8) * 2;
                all_l[h] += x[1] * exp2_fast(x[0] - b);
            }
            mine[h] = exp2_fast(m[h] - b);
            m[h] = all_m[h];
            l[h] = all_l[h];
        }
#pragma unroll
        for (int n = 0; n < DP / 8; ++n)
#pragma unroll
            for (int h = 0; h < 2; ++h)
                *reinterpret_cast<float2 *>(eo + (warp * 16 + g + h * 8) * (DP + 8) + n * 8 + 2 * t) =
                    make_float2(o[n][2 * h] * mine[h], o[n][2 * h + 1] * mine[h]);
        __syncthreads();
        // every thread adds a share of the columns
        for (int i = tid; i < WM * 16 * (DP / 4); i += kAtThreads) {
            const int r = i / (DP / 4), c = i % (DP / 4) * 4;
            if (r >= it.nrows || c >= hd) continue;
            float4 v = make_float4(0, 0, 0, 0);
#pragma unroll
            for (int k = 0; k < KW; ++k) {
                const float4 x = *reinterpret_cast<const float4 *>(eo + ((k * WM + r / 16) * 16 + r % 16) * (DP + 8) + c);
                v.x += x.x; v.y += x.y; v.z += x.z; v.w += x.w;
            }
            const long long row = it.row0 + r, out_row = (row / G) * a.n_heads + it.kh * G + row % G;
            *reinterpret_cast<float4 *>(o_part + ((long long)it.slot * rows_total + out_row) * hd + c) = v;
        }
        if (wk == 0 && t == 0)
#pragma unroll
            for (int h = 0; h < 2; ++h)
                if (rloc[h] < it.nrows) {
                    const long long row = it.row0 + rloc[h], out_row = (row / G) * a.n_heads + it.kh * G + row % G;
                    ml_part[(long long)it.slot * rows_total + out_row] = make_float2(m[h], l[h]);
                }
    } else {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            if (rloc[h] >= it.nrows) continue;
            const long long row = it.row0 + rloc[h], out_row = (row / G) * a.n_heads + it.kh * G + row % G;
            float *dst = o_part + ((long long)it.slot * rows_total + out_row) * hd;
#pragma unroll
            for (int n = 0; n < DP / 8; ++n)
                if (n * 8 < hd) *reinterpret_cast<float2 *>(dst + n * 8 + 2 * t) = make_float2(o[n][2 * h], o[n][2 * h + 1]);
            if (t == 0) ml_part[(long long)it.slot * rows_total + out_row] = make_float2(m[h], l[h]);
        }
    }
}

template <int DP>
constexpr size_t attention_smem() { return (size_t)kAtStages * 2 * kAtTile * (DP * 2 + 16) + (kAtStages + 1) * kAtTile * 8; }

template <class D, int DP>
__global__ void __launch_bounds__(kAtThreads, 2)
attention_items_kernel(const AttentionArgs a, const AttentionPlan p, float *o_part, float2 *ml_part)
{
    extern __shared__ __align__(16) unsigned char smem[];
    pdl_begin();
    const int G = a.n_heads / a.n_kv;
    AttentionItem it;
    int wm;
    long long x = blockIdx.x;
    if (x < p.pre_items) {
        // row tiles of the same keys are neighbours: they find them in the L2
        const long long rows = a.n_seq * a.n_q * G;
        const int rt = (int)(x % p.pre_rt);
        x /= p.pre_rt;
        const int s = (int)(x % p.pre_splits);
        it.kh = (int)(x / p.pre_splits);
        const long long tiles = (a.prefix_len + kAtTile - 1) / kAtTile;
        it.pages = a.prefix_pages;
        it.k0 = tiles * s / p.pre_splits * kAtTile;
        it.k1 = min(a.prefix_len, tiles * (s + 1) / p.pre_splits * kAtTile);
        it.limit0 = 0;
        it.row0 = (long long)rt * 16 * p.pre_wm;
        it.nrows = (int)min(rows - it.row0, 16ll * p.pre_wm);
        it.slot = s;
        it.own = false;
        wm = p.pre_wm;
    } else {
        x -= p.pre_items;
        const int s = (int)(x % p.own_splits);
        x /= p.own_splits;
        const int rt = (int)(x % p.own_rt);
        x /= p.own_rt;
        it.kh = (int)(x % a.n_kv);
        const long long b = x / a.n_kv;
        const long long len = own_length(a, b, threadIdx.x == 0 && s == 0 && rt == 0 && it.kh == 0);
        const long long tiles = (len + kAtTile - 1) / kAtTile;
        const int splits = own_splits_of(tiles, p.own_splits, p.own_chunk);
        if (s >= splits) return;
        it.pages = a.page_table + b * a.ld_table;
        it.k0 = tiles * s / splits * kAtTile;
        it.k1 = min(len, tiles * (s + 1) / splits * kAtTile);
        it.limit0 = len - (a.n_q - 1);
        it.row0 = b * a.n_q * G + (long long)rt * 16 * p.own_wm;
        it.nrows = (int)min((long long)a.n_q * G - (long long)rt * 16 * p.own_wm, 16ll * p.own_wm);
        it.slot = p.pre_splits + s;
        it.own = true;
        wm = p.own_wm;
    }
    if (wm == 1) attention_item<D, DP, 1>(a, it, o_part, ml_part, p.rows, smem);
    else if (wm == 2) attention_item<D, DP, 2>(a, it, o_part, ml_part, p.rows, smem);
    else attention_item<D, DP, 4>(a, it, o_part, ml_part, p.rows, smem);
}

// One warp per row (token, head): the slices' maxima and sums, then the weighted outputs.
template <class D>
__global__ void __launch_bounds__(128)
attention_join_kernel(const AttentionArgs a, const AttentionPlan p, const float *__restrict__ o_part, const float2 *__restrict__ ml_part)
{
    pdl_begin();
    const int lane = threadIdx.x & 31;
    const long long r = (long long)blockIdx.x * 4 + (threadIdx.x >> 5);
    if (r >= p.rows) return;
    const long long tok = r / a.n_heads, len = own_length(a, tok / a.n_q, false);
    const int n = p.pre_splits + own_splits_of((len + kAtTile - 1) / kAtTile, p.own_splits, p.own_chunk);
    float m = -CUDART_INF_F, l = 0.0f;
    for (int i = lane; i < n; i += 32) m = fmaxf(m, ml_part[(long long)i * p.rows + r].x);
    for (int x = 16; x > 0; x >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, x));
    const float base = m == -CUDART_INF_F ? 0.0f : m;
    float4 o = make_float4(0, 0, 0, 0);
    const bool in = lane * 4 < a.head_dim;
    for (int i = 0; i < n; ++i) {
        const float2 x = ml_part[(long long)i * p.rows + r];
        const float w = exp2_fast(x.x - base);
        l += w * x.y;
        if (in) {
            const float4 v = *reinterpret_cast<const float4 *>(o_part + ((long long)i * p.rows + r) * a.head_dim + lane * 4);
            o.x += w * v.x; o.y += w * v.y; o.z += w * v.z; o.w += w * v.w;
        }
    }
    if (in) {
        const float inv = l == 0.0f ? 0.0f : 1.0f / l;          // no key at all: zeros
        *reinterpret_cast<uint2 *>(a.out + tok * a.ldo + (r % a.n_heads) * a.head_dim + lane * 4) =
            make_uint2(D::encode2(o.x * inv, o.y * inv), D::encode2(o.z * inv, o.w * inv));
    }
}

template <class D, int DP>
static aweq_status items_launch(const AttentionArgs &a, const AttentionPlan &p, float *o_part, float2 *ml_part, cudaStream_t stream)
{
    constexpr size_t smem = attention_smem<DP>();
    static_assert(4 * 16 * 2 * 4 + 4 * 16 * (DP + 8) * 4 <= smem, "the join reuses the stages");
    AWEQ_CUDA_OK(cudaFuncSetAttribute(attention_items_kernel<D, DP>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem));
    AWEQ_LAUNCH((attention_items_kernel<D, DP>), dim3((unsigned)(p.pre_items + p.own_items)), dim3(kAtThreads), smem, stream, a, p,
                o_part, ml_part);
    return AWEQ_OK;
}

template <class D>
static aweq_status attention_launch(const AttentionArgs &a, void *ws, cudaStream_t stream)
{
    const AttentionPlan p = attention_plan(a.prefix_len, a.max_own, a.n_seq, a.n_q, a.n_heads, a.n_kv, a.head_dim);
    if (p.pre_items + p.own_items > 0x7fffffffll) return AWEQ_ERR_SHAPE;
    float *o_part = reinterpret_cast<float *>(ws);
    float2 *ml_part = reinterpret_cast<float2 *>(reinterpret_cast<char *>(ws) + p.off_ml);
    if (p.pre_items + p.own_items > 0) {
        const aweq_status rc = p.dp == 64 ? items_launch<D, 64>(a, p, o_part, ml_part, stream)
                               : p.dp == 96 ? items_launch<D, 96>(a, p, o_part, ml_part, stream)
                                            : items_launch<D, 128>(a, p, o_part, ml_part, stream);
        if (rc != AWEQ_OK) return rc;
    }
    AWEQ_LAUNCH(attention_join_kernel<D>, dim3((unsigned)((p.rows + 3) / 4)), dim3(128), 0, stream, a, p, (const float *)o_part,
                (const float2 *)ml_part);
    return AWEQ_OK;
}

aweq_status run_prefix_attention(const AttentionArgs &a, aweq_dtype dt, void *ws, cudaStream_t stream)
{
    return dt == AWEQ_F16 ? attention_launch<F16>(a, ws, stream) : attention_launch<BF16>(a, ws, stream);
}

}  // namespace aweq
