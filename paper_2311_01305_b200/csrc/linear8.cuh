// Shared pieces of the 8-bit linear layer (aweq_linear_w8a8):
//   out[n,o] = Step^x_n Step^w_o acc + bias_o,  acc = sum_k (xq[n,k] - Z^x_n)(wq[o,k] - Z^w_o)
//            = S - Z^x cw_o - Z^w (rx_n - K Z^x),   S = sum_k xq wq,  rx_n = sum_k xq,  cw_o = sum_k wq.
// S comes from the tensor cores as unsigned 8-bit products added modulo 2^32.
#pragma once
#include "common.cuh"
#include "kernels.h"

namespace aweq {

// (kept out of the kernels' loops: 16 x 4096 x 12288 took 12.7 us with it inside, 12.5 with a call)
static __device__ __noinline__ float linear8_acc_wide(uint32_t S, int zx, uint32_t rx, int zw, uint32_t cw, uint32_t K, bool in64)
{
    if (in64) {
        const long long x = zx, w = zw;
        const unsigned long long u = rx - K * (unsigned long long)x;
        return (float)(long long)(S - (unsigned long long)x * cw - (unsigned long long)w * u);
    }
    const double u = (double)rx - (double)K * (double)zx;
    return (float)((double)S - (double)zx * (double)cw - (double)zw * u);
}
// acc from its parts.  With bx = max(|Z^x|, |255 - Z^x|) no |xq - Z^x| is larger than bx, likewise
// for w, so |acc| <= K bx bw.  Where that is below 2^31 (every pair of zero-points inside the code
// range up to K = 33025, and far beyond for zero-points near the middle) the parts may wrap and
// acc is still exact modulo 2^32, hence exact; below 2^62 the same holds of 64 bits.  Beyond, the parts are joined in
// binary64 (S itself is below 2^32 for K <= 65536), rounded where they pass 2^53.
__device__ __forceinline__ float linear8_acc(uint32_t S, int zx, uint32_t rx, int zw, uint32_t cw, uint32_t K, float bxK,
                                             float bw)
{
    if (bxK * bw < 2.147e9f)
        return (float)(int)(S - (uint32_t)zx * cw - (uint32_t)zw * (rx - K * (uint32_t)zx));
    return linear8_acc_wide(S, zx, rx, zw, cw, K, bxK * bw < 4.6e18f);
}
__device__ __forceinline__ float linear8_reach(int z) { return fmaxf(fabsf((float)z), fabsf(255.0f - (float)z)); }

struct Linear8Args {
    const unsigned char *X, *W;
    long long ldx, ldw, ldo, N;
    const float *x_step, *w_step, *bias;
    const int *x_zp, *w_zp, *w_sum;
    int x_inc, w_inc;              // 1: a pair per row, 0: one pair for all rows
    int K, O;
    uint16_t *out;
    aweq_dev_status *st;
};

aweq_status run_linear8_stream(const Linear8Args &a, aweq_dtype dt, cudaStream_t stream);       // linear8.cu
aweq_status run_linear8(const Linear8Args &a, aweq_dtype dt, cudaStream_t stream);              // linear8_tc.cu: any of them

}  // namespace aweq
