// aweq_prefix_attention: n_q tokens per sequence over a shared prefix and each sequence's own keys.
#include <math_constants.h>

#include "common.cuh"
#include "kernels.h"

namespace aweq {

size_t prefix_attention_ws_bytes(const aweq_kv_cache *, long long, long long, long long, int, int) { return 256; }

// One warp per (token, head), one key at a time: running maximum, sum and output in binary32.
template <class D>
__global__ void __launch_bounds__(128) attention_kernel(const AttentionArgs a)
{
    pdl_begin();
    const int lane = threadIdx.x & 31;
    const long long r = (long long)blockIdx.x * 4 + (threadIdx.x >> 5), rows = a.n_seq * a.n_q * a.n_heads;
    if (r >= rows) return;
    const int h = (int)(r % a.n_heads), kh = h / (a.n_heads / a.n_kv);
    const long long tok = r / a.n_heads, b = tok / a.n_q;
    long long len = a.own_len[b];
    const long long most = min(a.max_own, a.pages_per_seq * a.page_size);
    if (len < 0 || len > most) {
        if (a.st && lane == 0 && h == 0 && tok % a.n_q == 0) atomicAdd(&a.st->out_of_range, 1ull);
        len = len < 0 ? 0 : most;
    }
    long long own = len - (a.n_q - 1 - tok % a.n_q);
    if (own < 0) own = 0;
    float q[4], o[4] = {0, 0, 0, 0}, m = -CUDART_INF_F, l = 0.0f;
#pragma unroll
    for (int i = 0; i < 4; ++i)
        q[i] = i * 32 + lane < a.head_dim ? D::one(a.q[tok * a.ldq + (long long)h * a.head_dim + i * 32 + lane]) * a.scale : 0.0f;
    for (long long j = 0; j < a.prefix_len + own; ++j) {
        const long long c = j < a.prefix_len ? j : j - a.prefix_len;
        const int *pages = j < a.prefix_len ? a.prefix_pages : a.page_table + b * a.ld_table;
        long long page = pages[c / a.page_size];
        if (page < 0 || page >= a.n_pages) {
            if (a.st && lane == 0) atomicAdd(&a.st->out_of_range, 1ull);
            page = 0;
        }
        const long long at = page * a.page_stride + (c % a.page_size) * a.token_stride + kh * a.head_stride;
        float s = 0.0f, v[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const bool in = i * 32 + lane < a.head_dim;
            if (in) s = __fmaf_rn(q[i], D::one(a.ck[at + i * 32 + lane]), s);
            v[i] = in ? D::one(a.cv[at + i * 32 + lane]) : 0.0f;
        }
        s = warp_sum(s);
        const float mn = fmaxf(m, s), f = __expf(m - mn), p = __expf(s - mn);
        l = l * f + p;
#pragma unroll
        for (int i = 0; i < 4; ++i) o[i] = o[i] * f + p * v[i];
        m = mn;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if (i * 32 + lane < a.head_dim)
            a.out[tok * a.ldo + (long long)h * a.head_dim + i * 32 + lane] = D::encode(l == 0.0f ? 0.0f : o[i] / l);
}

aweq_status run_prefix_attention(const AttentionArgs &a, aweq_dtype dt, void *, cudaStream_t stream)
{
    const long long blocks = (a.n_seq * a.n_q * a.n_heads + 3) / 4;
    if (dt == AWEQ_F16)
        AWEQ_LAUNCH(attention_kernel<F16>, dim3((unsigned)blocks), dim3(128), 0, stream, a);
    else
        AWEQ_LAUNCH(attention_kernel<BF16>, dim3((unsigned)blocks), dim3(128), 0, stream, a);
    return AWEQ_OK;
}

}  // namespace aweq
