// aweq_linear_w8a8 for few tokens, and the row sums of weight codes.
#include "linear8.cuh"

namespace aweq {

// Row sums of the codes, once per layer: one warp per row, a read of the codes.
__global__ void __launch_bounds__(256) code_sums_kernel(const unsigned char *Q, long long rows, long long cols, long long ld, int *out)
{
    pdl_begin();
    const int lane = threadIdx.x & 31;
    const long long row = (long long)blockIdx.x * 8 + (threadIdx.x >> 5);
    if (row >= rows) return;
    const uint4 *p = reinterpret_cast<const uint4 *>(Q + row * ld);
    uint32_t acc = 0;
    for (long long i = lane; i < cols / 16; i += 32) {
        const uint4 v = ld_stream(p + i);
        acc = __dp4a(v.x, 0x01010101u, acc);
        acc = __dp4a(v.y, 0x01010101u, acc);
        acc = __dp4a(v.z, 0x01010101u, acc);
        acc = __dp4a(v.w, 0x01010101u, acc);
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) acc += __shfl_xor_sync(0xffffffffu, acc, o);
    if (lane == 0) out[row] = (int)acc;
}

aweq_status run_code_sums(const unsigned char *codes, long long rows, long long cols, long long ld, int *sums,
                          cudaStream_t stream)
{
    AWEQ_LAUNCH(code_sums_kernel, dim3((unsigned)((rows + 7) / 8)), dim3(256), 0, stream, codes, rows, cols, ld, sums);
    return AWEQ_OK;
}

__device__ __forceinline__ void mma_u8(uint32_t (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0,
                                       uint32_t b1)
{
    asm volatile("mma.sync.aligned.m16n8k32.row.col.s32.u8.u8.s32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+r"(c[0]), "+r"(c[1]), "+r"(c[2]), "+r"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// Few tokens: the layer is a read of the weights.  A CTA owns 16 output channels (the 16 rows of an
// m16n8k32 tile) and 8 NT tokens; its eight warps take the row's 64-byte segments in turn.  A product is the
// same under any order of k that both operands share, so a lane loads 16 consecutive bytes of its
// two rows (lane % 4 picks the quarter of the segment) straight into the registers of two instructions
// and the same bytes of its token: no shared memory, no barrier until the warps' sums are added.  Bound by the start of a launch and the
// latency of the loads (1 x 768 x 768: 2.4 us on the device, a call of the binding 7.6), then by memory (1 x 4096 x 4096: 6.8 us).
template <int NT, class D>
__global__ void __launch_bounds__(256) linear8_stream_kernel(const Linear8Args p)
{
    pdl_begin();
    constexpr int kWarps = 8, U = NT <= 2 ? 4 : 2;
    __shared__ uint32_t part[kWarps][NT * 8][17];
    __shared__ uint32_t rsum[kWarps][NT * 8];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, g = lane >> 2, t = lane & 3;
    const int o0 = blockIdx.x * 16;
    const long long n0 = (long long)blockIdx.y * (NT * 8);
    // rows beyond the matrix read the last one; what they give is not written
    const unsigned char *wa = p.W + (long long)min(o0 + g, p.O - 1) * p.ldw + t * 16;
    const unsigned char *wb = p.W + (long long)min(o0 + g + 8, p.O - 1) * p.ldw + t * 16;
    const unsigned char *xt[NT];
#pragma unroll
    for (int i = 0; i < NT; ++i) xt[i] = p.X + min(n0 + i * 8 + g, p.N - 1) * p.ldx + t * 16;
    uint32_t acc[NT][4] = {}, rx[NT] = {};
    const int nseg = (p.K + 63) / 64;
    for (int s0 = warp; s0 < nseg; s0 += kWarps * U) {
        uint4 a[U], b[U], x[U][NT];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int k = (s0 + u * kWarps) * 64;
            const bool in = k + t * 16 < p.K;              // K is a multiple of 16: a quarter is all in or all out
            const uint4 zero = make_uint4(0, 0, 0, 0);
            a[u] = in ? ld_stream(wa + k) : zero;
            b[u] = in ? ld_stream(wb + k) : zero;
#pragma unroll
            for (int i = 0; i < NT; ++i) x[u][i] = in ? *reinterpret_cast<const uint4 *>(xt[i] + k) : zero;
        }
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int i = 0; i < NT; ++i) {
                mma_u8(acc[i], a[u].x, b[u].x, a[u].y, b[u].y, x[u][i].x, x[u][i].y);
                mma_u8(acc[i], a[u].z, b[u].z, a[u].w, b[u].w, x[u][i].z, x[u][i].w);
                rx[i] = __dp4a(x[u][i].x, 0x01010101u, rx[i]);
                rx[i] = __dp4a(x[u][i].y, 0x01010101u, rx[i]);
                rx[i] = __dp4a(x[u][i].z, 0x01010101u, rx[i]);
                rx[i] = __dp4a(x[u][i].w, 0x01010101u, rx[i]);
            }
    }
#pragma unroll
    for (int i = 0; i < NT; ++i) {
        part[warp][i * 8 + 2 * t][g] = acc[i][0];
        part[warp][i * 8 + 2 * t + 1][g] = acc[i][1];
        part[warp][i * 8 + 2 * t][g + 8] = acc[i][2];
        part[warp][i * 8 + 2 * t + 1][g + 8] = acc[i][3];
        rx[i] += __shfl_xor_sync(0xffffffffu, rx[i], 1);
        rx[i] += __shfl_xor_sync(0xffffffffu, rx[i], 2);
        if (t == 0) rsum[warp][i * 8 + g] = rx[i];
    }
    __syncthreads();
    for (int i = threadIdx.x; i < NT * 128; i += 256) {
        const int r = i >> 4, c = i & 15, o = o0 + c;
        const long long n = n0 + r;
        if (n >= p.N || o >= p.O) continue;
        uint32_t S = 0, rows = 0;
#pragma unroll
        for (int w = 0; w < kWarps; ++w) {
            S += part[w][r][c];
            rows += rsum[w][r];
        }
        const int zx = p.x_zp[n * p.x_inc], zw = p.w_zp[(long long)o * p.w_inc];
        const float v = linear8_acc(S, zx, rows, zw, (uint32_t)p.w_sum[o], (uint32_t)p.K, linear8_reach(zx) * (float)p.K,
                                    linear8_reach(zw));
        const float y = __fmaf_rn(v * p.x_step[n * p.x_inc], p.w_step[(long long)o * p.w_inc], p.bias ? p.bias[o] : 0.0f);
        p.out[n * p.ldo + o] = D::encode(y);
    }
}

template <class D>
static aweq_status stream_launch(const Linear8Args &a, cudaStream_t stream)
{
    const int nt = a.N <= 8 ? 1 : a.N <= 16 ? 2 : 4;
    const dim3 grid((unsigned)((a.O + 15) / 16), (unsigned)((a.N + 8 * nt - 1) / (8 * nt)));     // (few tokens: two rows at most)
    if (nt == 1)
        AWEQ_LAUNCH((linear8_stream_kernel<1, D>), grid, dim3(256), 0, stream, a);
    else if (nt == 2)
        AWEQ_LAUNCH((linear8_stream_kernel<2, D>), grid, dim3(256), 0, stream, a);
    else
        AWEQ_LAUNCH((linear8_stream_kernel<4, D>), grid, dim3(256), 0, stream, a);
    return AWEQ_OK;
}

aweq_status run_linear8_stream(const Linear8Args &a, aweq_dtype dt, cudaStream_t stream)
{
    return dt == AWEQ_F16 ? stream_launch<F16>(a, stream) : stream_launch<BF16>(a, stream);
}

}  // namespace aweq
