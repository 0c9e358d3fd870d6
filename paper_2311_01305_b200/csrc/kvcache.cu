// Rotary tables and the paged cache: aweq_rope_table, aweq_kv_append.
#include <math.h>

#include "common.cuh"
#include "kernels.h"

namespace aweq {

struct RopeArgs {
    double theta, factor, original_len, low, high, attention;
    int rd, scaling;
};

// One thread per (position, pair); everything in binary64, so the angle p f_i keeps 1e-16 of itself
// even at positions where a binary32 product is off by a visible part of a turn.
__global__ void __launch_bounds__(256) rope_table_kernel(const RopeArgs a, long long n_pos, float *__restrict__ table)
{
    pdl_begin();
    const int half = a.rd / 2;
    const double two_pi = 6.283185307179586;
    for (long long i = (long long)blockIdx.x * 256 + threadIdx.x; i < n_pos * half; i += (long long)gridDim.x * 256) {
        const long long p = i / half;
        const int j = (int)(i % half);
        double f = pow(a.theta, -2.0 * j / a.rd);
        if (a.scaling == AWEQ_ROPE_LINEAR) f /= a.factor;
        if (a.scaling == AWEQ_ROPE_BANDS) {
            const double turns = a.original_len * f / two_pi;
            const double keep = fmin(fmax((turns - a.low) / (a.high - a.low), 0.0), 1.0);
            f *= keep + (1.0 - keep) / a.factor;
        }
        double s, c;
        sincos((double)p * f, &s, &c);
        table[p * a.rd + j] = (float)(c * a.attention);
        table[p * a.rd + half + j] = (float)(s * a.attention);
    }
}

aweq_status run_rope_table(const aweq_rope *r, long long n_pos, float *table, cudaStream_t stream)
{
    RopeArgs a = {r->theta, r->factor, r->original_len, r->low, r->high, r->attention, r->rotary_dim, r->scaling};
    if (a.scaling == AWEQ_ROPE_BASE) a.theta *= pow(a.factor, (double)a.rd / (a.rd - 2));
    long long blocks = (n_pos * (a.rd / 2) + 255) / 256;
    if (blocks > kSmCount * 8) blocks = kSmCount * 8;
    AWEQ_LAUNCH(rope_table_kernel, dim3((unsigned)blocks), dim3(256), 0, stream, a, n_pos, table);
    return AWEQ_OK;
}

// ------------------------------------------------------------------ append
// Where token t goes, and whether it may.
struct AppendPlace {
    long long at;                // element of the pool (before the head) or -1: not stored
    int pos;
    bool turn_ok;                // position inside the table (or no rotation)
};
__device__ __forceinline__ AppendPlace append_place(const KvAppendArgs &a, long long t, bool count)
{
    AppendPlace w;
    w.pos = a.pos[t];
    w.turn_ok = !a.rope || (w.pos >= 0 && w.pos < a.n_pos);
    w.at = -1;
    if (a.slot) {
        const long long slot = a.slot[t];
        if (slot < 0) {                                         // no token
            w.turn_ok = false;
            return w;
        }
        const bool out = !w.turn_ok || slot >= a.n_pages * a.page_size;
        if (out && count && a.st) atomicAdd(&a.st->out_of_range, 1ull);
        if (!out) {
            const long long page = slot >> 32 ? slot / a.page_size : (long long)((uint32_t)slot / (uint32_t)a.page_size);
            w.at = page * a.page_stride + (slot - page * a.page_size) * a.token_stride;
        }
        return w;
    }
    const long long s = a.seq ? a.seq[t] : t, c = (long long)w.pos - a.first;
    bool bad = !w.turn_ok || s < 0 || s >= a.n_seq;
    if (!bad && c >= 0) {
        const unsigned in_seq = (unsigned)c / (unsigned)a.page_size, row = (unsigned)c % (unsigned)a.page_size;
        bad = in_seq >= a.pages_per_seq;
        if (!bad) {
            const long long page = a.page_table[s * a.ld_table + in_seq];
            bad = page < 0 || page >= a.n_pages;
            if (!bad) w.at = page * a.page_stride + (long long)row * a.token_stride;
        }
    }
    if (bad && count && a.st) atomicAdd(&a.st->out_of_range, 1ull);
    return w;
}
// source and destination of head h (queries, keys, values in this order) of token t; false: nothing to do
__device__ __forceinline__ bool append_head(const KvAppendArgs &a, const AppendPlace &w, long long t, int h, const uint16_t **src,
                                            uint16_t **dst)
{
    if (h < a.n_heads) {
        *src = a.q + t * a.ldq + (long long)h * a.head_dim;
        *dst = a.q_out + t * a.ld_qout + (long long)h * a.head_dim;
        return true;
    }
    const bool value = h >= a.n_heads + a.n_kv;
    const int kh = h - a.n_heads - (value ? a.n_kv : 0);
    *src = value ? a.v + t * a.ldv + (long long)kh * a.head_dim : a.k + t * a.ldk + (long long)kh * a.head_dim;
    *dst = (value ? a.cv : a.ck) + w.at + kh * a.head_stride;
    return w.at >= 0;
}

// 16-byte accesses.  The pass is a copy: what bounds it is memory, and before that the loads under way.  A warp
// takes one token and a run of its heads, a lane the same two 16-byte pieces of every head it gets (the two
// halves of eight pairs, or 16 neighbouring elements when interleaved), so cos and sin are read once per
// token and stay in registers, and four heads' loads are issued before the first is used.  Measured: 26624 tokens of 40 + 2 x 8 heads of
// 128, 138 us, 5.64 TB/s (a copy: 6.46); 64 tokens 3.8 us on the device (a call of the binding 10.5), three dependent loads (position and
// sequence, page, row) after the start, of which only the stores need the first two.  By slots: 384 tokens of 32 + 2 x 8 heads of 128 5.8 us in a
// row, 40000 of them 172 us, 5.7 TB/s.
template <class D, bool INTER>
__global__ void __launch_bounds__(256)
kv_append_kernel(const KvAppendArgs a, int segments)
{
    pdl_begin();
    const int lane = threadIdx.x & 31;
    const long long w = (long long)blockIdx.x * 8 + (threadIdx.x >> 5), t = w / segments;
    if (t >= a.n_tokens) return;
    const int seg = (int)(w % segments);
    const int units = (a.head_dim + 15) / 16, per = 32 / units, u = lane % units, sub = lane / units;
    const int heads = a.n_heads + 2 * a.n_kv, turned = a.n_heads + a.n_kv;
    const int h0 = (int)((long long)heads * seg / segments), h1 = (int)((long long)heads * (seg + 1) / segments);
    const AppendPlace place = append_place(a, t, lane == 0 && seg == 0);
    if (sub >= per) return;
    const int rd = a.rd;
    // the lane's two pieces, in elements of the head
    const bool turn0 = u * 16 < rd, turn1 = INTER ? u * 16 + 8 < rd : turn0;
    const int e0 = !INTER && turn0 ? u * 8 : u * 16, e1 = !INTER && turn0 ? u * 8 + rd / 2 : u * 16 + 8;
    float co[8], si[8];
    if (turn0 && place.turn_ok) {
        const float *cs = a.rope + (long long)place.pos * rd + u * 8;
        load8(cs, co);
        if (!INTER || turn1) load8(cs + rd / 2, si);
        else {                                                  // the last four pairs of an interleaved head: no more than they
            const float4 s4 = ldg_f4(cs + rd / 2);
            si[0] = s4.x; si[1] = s4.y; si[2] = s4.z; si[3] = s4.w;
        }
    }
    constexpr int U = 4;
    for (int hb = h0 + sub; hb < h1; hb += per * U) {
        uint4 x[U], y[U];
        uint16_t *dst[U];
        bool on[U];
#pragma unroll
        for (int i = 0; i < U; ++i) {
            const uint16_t *src;
            const int h = hb + i * per;
            on[i] = h < h1 && append_head(a, place, t, h, &src, &dst[i]);
            // a plain copy of values and of what is not turned keeps the same two pieces of the head
            const bool plain = !INTER && turn0 && h >= turned;
            if (on[i]) {
                x[i] = *reinterpret_cast<const uint4 *>(src + (plain ? u * 16 : e0));
                if (plain || e1 < a.head_dim) y[i] = *reinterpret_cast<const uint4 *>(src + (plain ? u * 16 + 8 : e1));
            }
        }
#pragma unroll
        for (int i = 0; i < U; ++i) {
            if (!on[i]) continue;
            const int h = hb + i * per;
            if (h >= turned) {
                *reinterpret_cast<uint4 *>(dst[i] + u * 16) = x[i];
                if (u * 16 + 8 < a.head_dim) *reinterpret_cast<uint4 *>(dst[i] + u * 16 + 8) = y[i];
                continue;
            }
            if (!place.turn_ok) {
                x[i] = y[i] = make_uint4(0, 0, 0, 0);
            } else if (!INTER && turn0) {
                float f[8], g[8];
                widen8<D>(x[i], f);
                widen8<D>(y[i], g);
                uint32_t *px = &x[i].x, *py = &y[i].x;
#pragma unroll
                for (int j = 0; j < 8; j += 2) {
                    px[j / 2] = D::encode2(__fmaf_rn(f[j], co[j], -(g[j] * si[j])), __fmaf_rn(f[j + 1], co[j + 1], -(g[j + 1] * si[j + 1])));
                    py[j / 2] = D::encode2(__fmaf_rn(f[j], si[j], g[j] * co[j]), __fmaf_rn(f[j + 1], si[j + 1], g[j + 1] * co[j + 1]));
                }
            } else if (INTER) {
#pragma unroll
                for (int half = 0; half < 2; ++half) {
                    if (!(half ? turn1 : turn0)) continue;
                    uint4 &v = half ? y[i] : x[i];
                    float f[8];
                    widen8<D>(v, f);
                    uint32_t *pv = &v.x;
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const float c = co[half * 4 + j], s = si[half * 4 + j];
                        pv[j] = D::encode2(__fmaf_rn(f[2 * j], c, -(f[2 * j + 1] * s)), __fmaf_rn(f[2 * j], s, f[2 * j + 1] * c));
                    }
                }
            }
            *reinterpret_cast<uint4 *>(dst[i] + e0) = x[i];
            if (e1 < a.head_dim) *reinterpret_cast<uint4 *>(dst[i] + e1) = y[i];
        }
    }
}

// Element by element, for rows or rotations that 16-byte pieces do not fit: the same formulas, several times slower (the first of the
// two cases above took 657 us in this form).
template <class D>
__global__ void __launch_bounds__(256) kv_append_elements_kernel(const KvAppendArgs a)
{
    pdl_begin();
    const long long t = blockIdx.x;
    const int d = a.head_dim, half = a.rd / 2;
    const AppendPlace place = append_place(a, t, threadIdx.x == 0 && blockIdx.y == 0);
    const float *cs = a.rope + (place.turn_ok ? (long long)place.pos : 0) * a.rd;
    const int heads = a.n_heads + 2 * a.n_kv;
    for (int i = blockIdx.y * 256 + threadIdx.x; i < heads * d; i += gridDim.y * 256) {
        const int h = i / d, e = i % d;
        const uint16_t *src;
        uint16_t *dst;
        if (!append_head(a, place, t, h, &src, &dst)) continue;
        if (h >= a.n_heads + a.n_kv || (e >= a.rd && place.turn_ok)) {
            dst[e] = src[e];
            continue;
        }
        if (!place.turn_ok) {
            dst[e] = 0;
            continue;
        }
        // the thread of a pair's first element turns both
        if (a.interleaved ? e & 1 : e >= half) continue;
        const int j = a.interleaved ? e / 2 : e, e2 = a.interleaved ? e + 1 : e + half;
        const float x = D::one(src[e]), y = D::one(src[e2]), co = cs[j], si = cs[half + j];
        dst[e] = D::encode(__fmaf_rn(x, co, -(y * si)));
        dst[e2] = D::encode(__fmaf_rn(x, si, y * co));
    }
}

static bool append_vectors(const KvAppendArgs &a)
{
    auto fits = [](const void *p, long long ld) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0 && ld % 8 == 0; };
    if (!fits(a.k, a.ldk) || !fits(a.v, a.ldv)) return false;
    if (a.n_heads && (!fits(a.q, a.ldq) || !fits(a.q_out, a.ld_qout))) return false;
    return !a.rope || (fits(a.rope, 0) && a.rd % (a.interleaved ? 8 : 16) == 0);
}

template <class D>
static aweq_status append_launch(const KvAppendArgs &a, cudaStream_t stream)
{
    const int heads = a.n_heads + 2 * a.n_kv;
    if (!append_vectors(a)) {
        const long long elems = (long long)heads * a.head_dim;
        AWEQ_LAUNCH(kv_append_elements_kernel<D>, dim3((unsigned)a.n_tokens, (unsigned)((elems + 2047) / 2048)), dim3(256), 0, stream, a);
        return AWEQ_OK;
    }
    // a token's heads over several warps while the tokens alone do not give every SM 32 of them
    const int per = 32 / ((a.head_dim + 15) / 16), most = (heads + per - 1) / per;
    long long segments = (kSmCount * 32 + a.n_tokens - 1) / a.n_tokens;
    if (segments > most) segments = most;
    const dim3 grid((unsigned)((a.n_tokens * segments + 7) / 8));
    if (a.interleaved && a.rope)
        AWEQ_LAUNCH((kv_append_kernel<D, true>), grid, dim3(256), 0, stream, a, (int)segments);
    else
        AWEQ_LAUNCH((kv_append_kernel<D, false>), grid, dim3(256), 0, stream, a, (int)segments);
    return AWEQ_OK;
}

aweq_status run_kv_append(const KvAppendArgs &a, aweq_dtype dt, cudaStream_t stream)
{
    return dt == AWEQ_F16 ? append_launch<F16>(a, stream) : append_launch<BF16>(a, stream);
}

}  // namespace aweq
