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
template <class D>
__global__ void __launch_bounds__(256) kv_append_kernel(const KvAppendArgs a)
{
    pdl_begin();
    const long long t = blockIdx.x;
    const int d = a.head_dim, half = a.rope ? a.rd / 2 : 0;
    const int pos = a.pos[t];
    const bool turn_ok = !a.rope || (pos >= 0 && pos < a.n_pos);
    const long long s = a.seq ? a.seq[t] : t, c = (long long)pos - a.first;
    long long page = -1;
    bool bad = !turn_ok || s < 0 || s >= a.n_seq;
    if (!bad && c >= 0) {
        if (c / a.page_size >= a.pages_per_seq) bad = true;
        else {
            page = a.page_table[s * a.ld_table + c / a.page_size];
            if (page < 0 || page >= a.n_pages) { bad = true; page = -1; }
        }
    }
    if (bad && a.st && threadIdx.x == 0 && blockIdx.y == 0) atomicAdd(&a.st->out_of_range, 1ull);
    const float *cs = a.rope + (turn_ok ? (long long)pos : 0) * a.rd;
    const int heads = a.n_heads + 2 * a.n_kv;
    const long long at = page * a.page_stride + (c % a.page_size) * a.token_stride;
    for (int i = blockIdx.y * 256 + threadIdx.x; i < heads * d; i += gridDim.y * 256) {
        const int h = i / d, e = i % d;
        const uint16_t *src;
        uint16_t *dst;
        if (h < a.n_heads) {
            src = a.q + t * a.ldq + (long long)h * d;
            dst = a.q_out + t * a.ld_qout + (long long)h * d;
        } else {
            const int kh = (h - a.n_heads) % a.n_kv;
            const bool value = h >= a.n_heads + a.n_kv;
            if (page < 0) continue;
            src = value ? a.v + t * a.ldv + (long long)kh * d : a.k + t * a.ldk + (long long)kh * d;
            dst = (value ? a.cv : a.ck) + at + kh * a.head_stride;
            if (value) { dst[e] = src[e]; continue; }
        }
        if (e >= 2 * half) { dst[e] = src[e]; continue; }
        // the thread of a pair's first element turns both
        const int j = a.interleaved ? e / 2 : e;
        const bool first = a.interleaved ? (e & 1) == 0 : e < half;
        if (!first) continue;
        const int e2 = a.interleaved ? e + 1 : e + half;
        if (!turn_ok) { dst[e] = dst[e2] = 0; continue; }
        const float x = D::one(src[e]), y = D::one(src[e2]), co = cs[j], si = cs[half + j];
        dst[e] = D::encode(__fmaf_rn(x, co, -(y * si)));
        dst[e2] = D::encode(__fmaf_rn(x, si, y * co));
    }
}

aweq_status run_kv_append(const KvAppendArgs &a, aweq_dtype dt, cudaStream_t stream)
{
    const long long elems = (long long)(a.n_heads + 2 * a.n_kv) * a.head_dim;
    const unsigned gy = (unsigned)((elems + 2047) / 2048);
    const dim3 grid((unsigned)a.n_tokens, gy);
    if (dt == AWEQ_F16)
        AWEQ_LAUNCH(kv_append_kernel<F16>, grid, dim3(256), 0, stream, a);
    else
        AWEQ_LAUNCH(kv_append_kernel<BF16>, grid, dim3(256), 0, stream, a);
    return AWEQ_OK;
}

}  // namespace aweq
