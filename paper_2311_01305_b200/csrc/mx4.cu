// aweq_quant_mx4 and aweq_dequant_mx4: 16-bit rows to microscaled 4-bit codes and back.
#include "mx4.cuh"

namespace aweq {

// eight binary32 values as eight e2m1 elements (round to nearest even, saturating at 6)
__device__ __forceinline__ uint32_t e2m1_encode8(const float2 *v)
{
    uint32_t r;
    asm("{\n\t.reg .b8 a, b, c, d;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 a, %2, %1;\n\tcvt.rn.satfinite.e2m1x2.f32 b, %4, %3;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 c, %6, %5;\n\tcvt.rn.satfinite.e2m1x2.f32 d, %8, %7;\n\t"
        "mov.b32 %0, {a, b, c, d};\n\t}"
        : "=r"(r) : "f"(v[0].x), "f"(v[0].y), "f"(v[1].x), "f"(v[1].y), "f"(v[2].x), "f"(v[2].y), "f"(v[3].x), "f"(v[3].y));
    return r;
}
__device__ __forceinline__ void e2m1_decode8(uint32_t codes, float *v)
{
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        // (a byte at a time: unpacked by one mov from a word that the same kernel had packed, the upper two came out as zeros)
        uint32_t h;
        asm("{\n\t.reg .b8 a;\n\tcvt.u8.u32 a, %1;\n\tcvt.rn.f16x2.e2m1x2 %0, a;\n\t}" : "=r"(h) : "r"(codes >> (8 * i)));
        const float2 f = __half22float2(F16::from_bits(h));
        v[2 * i] = f.x;
        v[2 * i + 1] = f.y;
    }
}
__device__ __forceinline__ uint32_t e4m3_encode(float v)
{
    uint16_t r;
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(0.0f), "f"(v));
    return r & 0xffu;
}
__device__ __forceinline__ float e4m3_decode(uint32_t b)
{
    uint32_t h;
    asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h) : "h"((uint16_t)b));
    return __half22float2(F16::from_bits(h)).x;
}

struct Mx4QuantArgs {
    const uint16_t *X;
    long long rows, ld, row_tiles;
    int cols, chunks, padded;                  // chunks of 16 columns, and those of whole groups of 256
    const float *scale, *mu;
    unsigned char *codes, *scales;
    float *row_step, *epsmu;
    aweq_dev_status *st;
};

struct Mx4Chunk { uint4 a, b; };               // 16 elements
__device__ __forceinline__ Mx4Chunk mx4_load(const Mx4QuantArgs &a, long long row, int chunk)
{
    Mx4Chunk c = {make_uint4(0, 0, 0, 0), make_uint4(0, 0, 0, 0)};
    if (row < a.rows && chunk < a.chunks) {
        // (read once; no invariant loads, since the launch that writes X may still run when this one starts)
        const uint16_t *p = a.X + row * a.ld + chunk * 16;
        asm volatile("ld.global.L1::no_allocate.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(c.a.x), "=r"(c.a.y), "=r"(c.a.z), "=r"(c.a.w) : "l"(p));
        asm volatile("ld.global.L1::no_allocate.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(c.b.x), "=r"(c.b.y), "=r"(c.b.z), "=r"(c.b.w) : "l"(p + 8));
    }
    return c;
}
// the elements times the columns' factors, two at a time
struct Mx4Scale { float2 f[8]; };
__device__ __forceinline__ Mx4Scale mx4_scale(const float *scale, int chunk, bool in)
{
    Mx4Scale m;
#pragma unroll
    for (int i = 0; i < 8; i += 2) {
        const float4 s = scale && in ? *reinterpret_cast<const float4 *>(scale + chunk * 16 + 2 * i) : make_float4(1.0f, 1.0f, 1.0f, 1.0f);
        m.f[i] = make_float2(s.x, s.y);
        m.f[i + 1] = make_float2(s.z, s.w);
    }
    return m;
}
template <class D>
__device__ __forceinline__ void mx4_values(const Mx4Chunk &c, const Mx4Scale &m, float2 (&v)[8])
{
    const uint32_t w[8] = {c.a.x, c.a.y, c.a.z, c.a.w, c.b.x, c.b.y, c.b.z, c.b.w};
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = __fmul2_rn(D::to_float2(D::from_bits(w[i])), m.f[i]);
}
// largest magnitude, as bits (infinities and NaN on top)
__device__ __forceinline__ uint32_t mx4_top(const float2 (&v)[8])
{
    float top = 0.0f;
#pragma unroll
    for (int i = 0; i < 8; ++i) asm("max.NaN.abs.f32 %0, %1, %2, %3;" : "=f"(top) : "f"(top), "f"(v[i].x), "f"(v[i].y));
    return __float_as_uint(top) & 0x7fffffffu;
}

//   v = x s_j,  step from the block's (and row's) largest |v|,  code = rn_e2m1(v / step): two operations on the values, one pass over X.
// A CTA takes a row, a thread V chunks of 16 columns; rows go round-robin over the grid with the next row's loads in flight.
// The factors of a thread's columns stay in registers where it has one chunk; its values do between their maximum and their codes.
// The steps are binary32, the one rounding is the element's (and, E4M3, the scale's).  Bound by memory, and close behind by its
// instructions (70 % of the issue slots): 11008 x 4096 to blocks of 16 in 26.5 us, 4.4 TB/s; 16 x 5120 3.2 us, all latency.  Loads of 32
// bytes in the place of two of 16 were slower (30 us: the registers wait for the later half).
template <class D, int FMT, int V, bool EPS>
__global__ void __launch_bounds__(V == 1 ? 512 : 1024)
mx4_quant_kernel(const Mx4QuantArgs a)
{
    __shared__ uint32_t sh_top[2][32];
    __shared__ float sh_eps[2][32];
    pdl_begin();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x >> 5;
    Mx4Scale kept;
    if (V == 1) kept = mx4_scale(a.scale, threadIdx.x, (int)threadIdx.x < a.chunks);
    auto factors = [&](int chunk) { return V == 1 ? kept : mx4_scale(a.scale, chunk, chunk < a.chunks); };
    constexpr bool kAhead = V <= 2;                             // (the registers hold the next row of up to 32768 columns too)
    Mx4Chunk x[V];
#pragma unroll
    for (int i = 0; i < V; ++i)
        if (kAhead) x[i] = mx4_load(a, blockIdx.x, threadIdx.x + i * blockDim.x);
    int turn = 0;
    for (long long row = blockIdx.x; row < a.rows; row += gridDim.x, turn ^= 1) {
        Mx4Chunk next[V];
#pragma unroll
        for (int i = 0; i < V; ++i) {
            if (kAhead) next[i] = mx4_load(a, row + gridDim.x, threadIdx.x + i * blockDim.x);
            else x[i] = mx4_load(a, row, threadIdx.x + i * blockDim.x);
        }
        float row_step = 1.0f;
        bool row_bad = false;
        if (FMT == AWEQ_MX4_E4M3) {
            uint32_t top = 0;
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const int chunk = threadIdx.x + i * blockDim.x;
                float2 v[8];
                mx4_values<D>(x[i], factors(chunk), v);
                top = max(top, mx4_top(v));
            }
            top = __reduce_max_sync(0xffffffffu, top);
            if (lane == 0) sh_top[turn][warp] = top;
            __syncthreads();
            top = __reduce_max_sync(0xffffffffu, lane < warps ? sh_top[turn][lane] : 0u);
            row_bad = top >= 0x7f800000u;
            row_step = row_bad ? __uint_as_float(0x7fffffffu) : __fmul_rn(__uint_as_float(top), 1.0f / 2688.0f);
            if (threadIdx.x == 0) {
                a.row_step[row] = row_step;
                if (row_bad && a.st) atomicAdd(&a.st->nonfinite, 1ull);
            }
        }
        float eps = 0.0f;
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const int chunk = threadIdx.x + i * blockDim.x;
            const bool in = chunk < a.chunks;
            float2 v[8];
            mx4_values<D>(x[i], factors(chunk), v);
            uint32_t top = mx4_top(v), byte;
            float step, inv;
            bool zero;
            if (FMT == AWEQ_MX4_E8M0) {
                top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
                zero = top >= 0x7f800000u;
                // floor(log2 top) - 2 and 127 more: the exponent field less two (subnormal maxima: the smallest scale)
                const int e = (int)(top >> 23) - 2;
                byte = e < 0 ? 0u : (uint32_t)e;
                step = byte ? __uint_as_float(byte << 23) : 5.877471754111438e-39f;
                inv = __uint_as_float((254u - byte) << 23);
                if (zero) {
                    byte = 0xffu;
                    if (in && (lane & 1) == 0 && a.st) atomicAdd(&a.st->nonfinite, 1ull);
                }
            } else {
                byte = row_bad ? 0u : e4m3_encode(__fdiv_rn(__uint_as_float(top), __fmul_rn(6.0f, row_step)));
                if (row_step == 0.0f) byte = 0u;
                step = __fmul_rn(e4m3_decode(byte), row_step);
                zero = !(step >= 1.17549435e-38f);
                if (zero) byte = 0u;
                inv = zero ? 0.0f : __frcp_rn(step);
            }
            // (inv is zero where the block becomes zeros; zero times an infinity or a NaN is none, but then every code is cleared)
            const float2 inv2 = make_float2(inv, inv);
            float2 y[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) y[j] = __fmul2_rn(v[j], inv2);
            uint2 codes = make_uint2(e2m1_encode8(y), e2m1_encode8(y + 4));
            if (zero) codes = make_uint2(0u, 0u);
            if (in) *reinterpret_cast<uint2 *>(a.codes + row * (a.cols / 2) + chunk * 8) = codes;
            // four blocks' scales to a word
            uint32_t word;
            if (FMT == AWEQ_MX4_E8M0) {
                word = byte << (8 * (chunk >> 1 & 3));
                word |= __shfl_xor_sync(0xffffffffu, word, 2);
                word |= __shfl_xor_sync(0xffffffffu, word, 4);
                if ((lane & 7) == 0 && chunk < a.padded)
                    *reinterpret_cast<uint32_t *>(a.scales + mx4_scale_at(row, chunk >> 1, a.row_tiles)) = word;
            } else {
                word = byte << (8 * (chunk & 3));
                word |= __shfl_xor_sync(0xffffffffu, word, 1);
                word |= __shfl_xor_sync(0xffffffffu, word, 2);
                if ((lane & 3) == 0 && chunk < a.padded)
                    *reinterpret_cast<uint32_t *>(a.scales + mx4_scale_at(row, chunk, a.row_tiles)) = word;
            }
            if (EPS && in) {
                float q[16];
                e2m1_decode8(codes.x, q);
                e2m1_decode8(codes.y, q + 8);
#pragma unroll
                for (int j = 0; j < 16; j += 4) {
                    const float4 m = *reinterpret_cast<const float4 *>(a.mu + chunk * 16 + j);
                    const float2 v0 = v[j / 2], v1 = v[j / 2 + 1];
                    eps = __fmaf_rn(__fmaf_rn(q[j], step, -v0.x), m.x, eps);
                    eps = __fmaf_rn(__fmaf_rn(q[j + 1], step, -v0.y), m.y, eps);
                    eps = __fmaf_rn(__fmaf_rn(q[j + 2], step, -v1.x), m.z, eps);
                    eps = __fmaf_rn(__fmaf_rn(q[j + 3], step, -v1.y), m.w, eps);
                }
            }
        }
        if (EPS) {
            eps = warp_sum(eps);
            if (lane == 0) sh_eps[turn][warp] = eps;
            __syncthreads();
            if (warp == 0) {
                eps = warp_sum(lane < warps ? sh_eps[turn][lane] : 0.0f);
                if (lane == 0) a.epsmu[row] = eps;
            }
        }
#pragma unroll
        for (int i = 0; i < V; ++i)
            if (kAhead) x[i] = next[i];
    }
}

template <class D, int FMT, int V>
static aweq_status quant_launch(const Mx4QuantArgs &a, unsigned threads, cudaStream_t stream)
{
    long long ctas = (long long)kSmCount * (2048 / threads > 8 ? 8 : 2048 / threads);
    if (ctas > a.rows) ctas = a.rows;
    if (a.epsmu)
        AWEQ_LAUNCH((mx4_quant_kernel<D, FMT, V, true>), dim3((unsigned)ctas), dim3(threads), 0, stream, a);
    else
        AWEQ_LAUNCH((mx4_quant_kernel<D, FMT, V, false>), dim3((unsigned)ctas), dim3(threads), 0, stream, a);
    return AWEQ_OK;
}
template <class D, int FMT>
static aweq_status quant_width(const Mx4QuantArgs &a, cudaStream_t stream)
{
    int v = a.padded <= 512 ? 1 : 2;
    while (a.padded > 1024 * v) ++v;
    const unsigned threads = (unsigned)((a.padded + 32 * v - 1) / (32 * v) * 32);
    switch (v) {
    case 1: return quant_launch<D, FMT, 1>(a, threads, stream);
    case 2: return quant_launch<D, FMT, 2>(a, threads, stream);
    case 3: return quant_launch<D, FMT, 3>(a, threads, stream);
    default: return quant_launch<D, FMT, 4>(a, threads, stream);
    }
}

aweq_status run_quant_mx4(const void *X, aweq_dtype dt, long long rows, long long cols, long long ld, const float *scale, int fmt,
                          unsigned char *codes, unsigned char *scales, float *row_step, const float *mu, float *epsmu,
                          aweq_dev_status *st, cudaStream_t stream)
{
    Mx4QuantArgs a = {reinterpret_cast<const uint16_t *>(X), rows, ld, mx4_row_tiles(cols, fmt), (int)cols, (int)(cols / 16),
                      (int)((cols + 255) / 256 * 16), scale, mu, codes, scales, row_step, epsmu, st};
    if (dt == AWEQ_F16)
        return fmt == AWEQ_MX4_E8M0 ? quant_width<F16, AWEQ_MX4_E8M0>(a, stream) : quant_width<F16, AWEQ_MX4_E4M3>(a, stream);
    return fmt == AWEQ_MX4_E8M0 ? quant_width<BF16, AWEQ_MX4_E8M0>(a, stream) : quant_width<BF16, AWEQ_MX4_E4M3>(a, stream);
}

// ------------------------------------------------------------------ back
// A thread has four chunks of 16 columns under way, each a load of 8 bytes and one sector written (as two halves: 31 us in the place of 21).
// Bound by memory: 11008 x 4096 from blocks of 16 in 20.9 us, 5.5 TB/s, 84 % of a copy.
template <class D, int FMT>
__global__ void __launch_bounds__(256)
mx4_dequant_kernel(const unsigned char *codes, const unsigned char *scales, const float *row_step, long long rows, int chunks,
                   long long row_tiles, uint16_t *out, long long ldo)
{
    pdl_begin();
    const long long total = rows * chunks, step = (long long)gridDim.x * 256;
    const bool wide = ldo % 16 == 0 && (reinterpret_cast<uintptr_t>(out) & 31) == 0;       // a chunk is a sector
    constexpr int U = 4;                                        // chunks of 16 columns under way
    for (long long i0 = (long long)blockIdx.x * 256 + threadIdx.x; i0 < total; i0 += U * step) {
        uint2 c[U];
        uint32_t byte[U];
        float r[U];
        uint16_t *dst[U];
#pragma unroll
        for (int k = 0; k < U; ++k) {
            const long long i = i0 + k * step;
            dst[k] = nullptr;
            if (i >= total) continue;
            const long long row = i >> 32 ? i / chunks : (long long)((uint32_t)i / (uint32_t)chunks);
            const int chunk = (int)(i - row * chunks);
            c[k] = *reinterpret_cast<const uint2 *>(codes + i * 8);
            byte[k] = scales[mx4_scale_at(row, FMT == AWEQ_MX4_E8M0 ? chunk >> 1 : chunk, row_tiles)];
            r[k] = FMT == AWEQ_MX4_E8M0 ? 1.0f : row_step[row];
            dst[k] = out + row * ldo + chunk * 16;
        }
#pragma unroll
        for (int k = 0; k < U; ++k) {
            if (!dst[k]) continue;
            float v[16], s;
            if (FMT == AWEQ_MX4_E8M0) s = byte[k] == 0xffu ? __uint_as_float(0x7fffffffu) : byte[k] ? __uint_as_float(byte[k] << 23) : 5.877471754111438e-39f;
            else s = e4m3_decode(byte[k]);
            e2m1_decode8(c[k].x, v);
            e2m1_decode8(c[k].y, v + 8);
            uint32_t o[8];
#pragma unroll
            for (int j = 0; j < 8; ++j)
                o[j] = FMT == AWEQ_MX4_E8M0 ? D::encode2(v[2 * j] * s, v[2 * j + 1] * s)
                                            : D::encode2(__fmul_rn(__fmul_rn(v[2 * j], s), r[k]), __fmul_rn(__fmul_rn(v[2 * j + 1], s), r[k]));
            if (wide)
                asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(dst[k]), "r"(o[0]), "r"(o[1]), "r"(o[2]), "r"(o[3]),
                             "r"(o[4]), "r"(o[5]), "r"(o[6]), "r"(o[7]) : "memory");
            else {
                uint4 *const to = reinterpret_cast<uint4 *>(dst[k]);
                to[0] = make_uint4(o[0], o[1], o[2], o[3]);
                to[1] = make_uint4(o[4], o[5], o[6], o[7]);
            }
        }
    }
}

template <class D, int FMT>
static aweq_status dequant_launch(const unsigned char *codes, const unsigned char *scales, const float *row_step, long long rows,
                                  long long cols, uint16_t *out, long long ldo, cudaStream_t stream)
{
    const long long chunks = cols / 16;
    long long ctas = (rows * chunks + 255) / 256;
    if (ctas > kSmCount * 8) ctas = kSmCount * 8;
    AWEQ_LAUNCH((mx4_dequant_kernel<D, FMT>), dim3((unsigned)ctas), dim3(256), 0, stream, codes, scales, row_step, rows, (int)chunks,
                mx4_row_tiles(cols, FMT), out, ldo);
    return AWEQ_OK;
}

aweq_status run_dequant_mx4(const unsigned char *codes, const unsigned char *scales, const float *row_step, int fmt, long long rows,
                            long long cols, void *out, aweq_dtype dt, long long ldo, cudaStream_t stream)
{
    uint16_t *o = reinterpret_cast<uint16_t *>(out);
    if (dt == AWEQ_F16)
        return fmt == AWEQ_MX4_E8M0 ? dequant_launch<F16, AWEQ_MX4_E8M0>(codes, scales, row_step, rows, cols, o, ldo, stream)
                                    : dequant_launch<F16, AWEQ_MX4_E4M3>(codes, scales, row_step, rows, cols, o, ldo, stream);
    return fmt == AWEQ_MX4_E8M0 ? dequant_launch<BF16, AWEQ_MX4_E8M0>(codes, scales, row_step, rows, cols, o, ldo, stream)
                                : dequant_launch<BF16, AWEQ_MX4_E4M3>(codes, scales, row_step, rows, cols, o, ldo, stream);
}

}  // namespace aweq
