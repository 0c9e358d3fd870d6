// The C ABI: host-side validation, workspace sizing and the composition of the
// six calibration steps into one layer pass.  No device memory is allocated
// here and nothing synchronises.
#include <atomic>
#include <cstdio>
#include <cstdlib>
#include <cstring>

#include "common.cuh"
#include "kernels.h"
#include "linear8.cuh"
#include "mx4.cuh"

namespace aweq {

static std::atomic<unsigned long long> g_launches{0};
static thread_local char g_cuda_error[256] = "";

void note_launch() { g_launches.fetch_add(1, std::memory_order_relaxed); }

aweq_status cuda_failed(cudaError_t e)
{
    snprintf(g_cuda_error, sizeof g_cuda_error, "%s: %s", cudaGetErrorName(e), cudaGetErrorString(e));
    return AWEQ_ERR_CUDA;
}

// AWEQ_LOG=1 in the environment: one line per entry-point call on stderr (shapes and the
// algorithmic bytes the call moves); read once.
static bool log_enabled()
{
    static const bool on = [] { const char *e = getenv("AWEQ_LOG"); return e && e[0] && e[0] != '0'; }();
    return on;
}
#define AWEQ_LOGF(...)                                       \
    do {                                                     \
        if (::aweq::log_enabled()) fprintf(stderr, "[aweq] " __VA_ARGS__); \
    } while (0)

static inline bool aligned(const void *p, size_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }
static inline size_t round256(size_t n) { return (n + 255) & ~(size_t)255; }

static aweq_status check_matrix(const void *M, aweq_dtype dt, long long rows, long long cols, long long ld,
                                bool allow_zero_rows)
{
    if (!M) return AWEQ_ERR_NULL;
    if (dt != AWEQ_F16 && dt != AWEQ_BF16) return AWEQ_ERR_DTYPE;
    if (cols <= 0 || (cols % 8) != 0 || cols > (1ll << 30)) return AWEQ_ERR_SHAPE;
    if (rows < 0 || (rows == 0 && !allow_zero_rows) || rows > (1ll << 40)) return AWEQ_ERR_SHAPE;
    if (ld < cols || (ld % 8) != 0) return AWEQ_ERR_ALIGN;
    if (!aligned(M, 16)) return AWEQ_ERR_ALIGN;
    return AWEQ_OK;
}

static aweq_status check_quant(int bits, int gran, int group, long long cols)
{
    if (bits < 2 || bits > 8) return AWEQ_ERR_BITS;
    if (gran != AWEQ_PER_TENSOR && gran != AWEQ_PER_ROW && gran != AWEQ_PER_GROUP) return AWEQ_ERR_UNSUPPORTED;
    if (gran == AWEQ_PER_GROUP) {
        if (group < 8 || group > 256 || (group & (group - 1)) != 0 || (cols % group) != 0) return AWEQ_ERR_GROUP;
    }
    return AWEQ_OK;
}

static aweq_status check_ws(void *ws, size_t ws_bytes, size_t need)
{
    if (need == 0) return AWEQ_OK;
    if (!ws || !aligned(ws, 256) || ws_bytes < need) return AWEQ_ERR_WORKSPACE;
    return AWEQ_OK;
}

static size_t eq_ws_bytes(long long rows, long long cols, int bits, int gran, int group)
{
    // per group of 128: the (window, row) partial sums of eps . E[x^]
    if (gran == AWEQ_PER_GROUP) return groupquant_supported(bits, group) ? round256(groupquant_ws_bytes(rows, cols)) : 0;
    if (gran != AWEQ_PER_TENSOR) return 0;
    // per-tensor: column extremes of W (2 x float[cols]) + lo/hi + the column-reduction scratch
    return round256((size_t)cols * 8) + 256 + colreduce_ws_bytes(rows, cols);
}

}  // namespace aweq

using namespace aweq;

extern "C" {

const char *aweq_strerror(aweq_status code)
{
    switch (code) {
    case AWEQ_OK: return "ok";
    case AWEQ_ERR_NULL: return "a required pointer is NULL";
    case AWEQ_ERR_SHAPE: return "bad shape (sizes must be positive, C_in a multiple of 8 and within the supported range)";
    case AWEQ_ERR_ALIGN: return "bad alignment (16-byte base pointers, row pitch a multiple of 8 elements and >= C_in)";
    case AWEQ_ERR_DTYPE: return "unknown 16-bit element type";
    case AWEQ_ERR_BITS: return "bit-width must be in 2..8";
    case AWEQ_ERR_GROUP: return "group size must be a power of two in [8, 256] that divides C_in";
    case AWEQ_ERR_WORKSPACE: return "workspace missing, misaligned (256 bytes) or too small";
    case AWEQ_ERR_CUDA: return "a CUDA call failed";
    case AWEQ_ERR_UNSUPPORTED: return "unsupported mode";
    case AWEQ_ERR_LIMIT: return "size beyond the built-in scratch of aweq_stats_static (C_in <= 16384)";
    }
    return "unknown status";
}

const char *aweq_last_cuda_error(void) { return g_cuda_error; }
int aweq_version(void) { return 101; }
unsigned long long aweq_launch_count(void) { return g_launches.load(std::memory_order_relaxed); }

aweq_status aweq_plan_query(int op, long long rows, long long cols, long long plan[8])
{
    if (!plan) return AWEQ_ERR_NULL;
    if (rows <= 0 || cols <= 0 || cols % 8 || cols > (1ll << 30)) return AWEQ_ERR_SHAPE;
    if (op == AWEQ_OP_STATS || op == AWEQ_OP_WRANGE) {
        colreduce_describe(rows, cols, plan);
        return AWEQ_OK;
    }
    if (op == AWEQ_OP_EQUALIZE_QUANTIZE || op == AWEQ_OP_QUANT_ACT)
        return rowquant_describe(rows, cols, op == AWEQ_OP_EQUALIZE_QUANTIZE, plan) ? AWEQ_OK : AWEQ_ERR_SHAPE;
    return AWEQ_ERR_UNSUPPORTED;
}

size_t aweq_workspace_bytes(int op, long long rows, long long cols, int bits, int gran, int group)
{
    if (cols <= 0 || rows < 0) return 0;
    switch (op) {
    case AWEQ_OP_STATS:
    case AWEQ_OP_WRANGE: return colreduce_ws_bytes(rows, cols);
    case AWEQ_OP_EQUALIZE_QUANTIZE: return eq_ws_bytes(rows, cols, bits, gran, group);
    default: return 0;
    }
}

aweq_status aweq_stats(const void *X, aweq_dtype dt, long long N, long long C_in, long long ldx, float *xmin,
                       float *xmax, float *xmean, double *xsum, long long *count, int accumulate, void *ws,
                       size_t ws_bytes, aweq_dev_status *st, void *stream)
{
    aweq_status rc = check_matrix(X, dt, N, C_in, ldx, true);
    if (rc != AWEQ_OK) return rc;
    if (!xmin || !xmax || !xmean) return AWEQ_ERR_NULL;
    if (accumulate && (!xsum || !count)) return AWEQ_ERR_NULL;
    if (!aligned(xmin, 16) || !aligned(xmax, 16) || !aligned(xmean, 4) || (xsum && !aligned(xsum, 8)))
        return AWEQ_ERR_ALIGN;
    rc = check_ws(ws, ws_bytes, colreduce_ws_bytes(N, C_in));
    if (rc != AWEQ_OK) return rc;
    AWEQ_LOGF("aweq_stats N=%lld C_in=%lld ld=%lld dtype=%d accumulate=%d bytes=%lld\n", N, C_in, ldx, (int)dt, accumulate,
              2 * N * C_in);
    return run_stats(X, dt, N, C_in, ldx, xmin, xmax, xmean, xsum, count, accumulate, ws, st, (cudaStream_t)stream);
}

aweq_status aweq_wrange(const void *W, aweq_dtype dt, long long C_out, long long C_in, long long ldw, float *wmin,
                        float *wmax, int accumulate, void *ws, size_t ws_bytes, aweq_dev_status *st, void *stream)
{
    aweq_status rc = check_matrix(W, dt, C_out, C_in, ldw, false);
    if (rc != AWEQ_OK) return rc;
    if (!wmin || !wmax) return AWEQ_ERR_NULL;
    rc = check_ws(ws, ws_bytes, colreduce_ws_bytes(C_out, C_in));
    if (rc != AWEQ_OK) return rc;
    AWEQ_LOGF("aweq_wrange C_out=%lld C_in=%lld accumulate=%d bytes=%lld\n", C_out, C_in, accumulate, 2 * C_out * C_in);
    return run_wrange(W, dt, C_out, C_in, ldw, wmin, wmax, accumulate, ws, st, (cudaStream_t)stream);
}

aweq_status aweq_factors(const float *xmin, const float *xmax, const float *xmean, const float *wmin,
                         const float *wmax, long long C_in, float *s, float *rinv, float *mu_hat, float *pX,
                         float *pW, double *scalars, aweq_dev_status *st, void *stream)
{
    if (!xmin || !xmax || !xmean || !wmin || !wmax || !s || !rinv || !mu_hat) return AWEQ_ERR_NULL;
    if (C_in <= 0 || C_in > (1ll << 20)) return AWEQ_ERR_SHAPE;
    return run_factors(xmin, xmax, xmean, wmin, wmax, C_in, s, rinv, mu_hat, pX, pW, scalars, st,
                       (cudaStream_t)stream);
}

aweq_status aweq_factors_absmax(const float *xmin, const float *xmax, const float *xmean, const float *wmin,
                                const float *wmax, long long C_in, float *s, float *rinv, float *mu_hat, float *pX,
                                float *pW, double *scalars, aweq_dev_status *st, void *stream)
{
    if (!xmin || !xmax || !xmean || !wmin || !wmax || !s || !rinv || !mu_hat) return AWEQ_ERR_NULL;
    if (C_in <= 0 || C_in > (1ll << 20)) return AWEQ_ERR_SHAPE;
    return run_factors(xmin, xmax, xmean, wmin, wmax, C_in, s, rinv, mu_hat, pX, pW, scalars, st,
                       (cudaStream_t)stream, 1);
}

static aweq_status equalize_quantize_impl(const void *W, aweq_dtype dt, long long C_out, long long C_in,
                                          long long ldw, const float *s, const float *mu_hat, int bits,
                                          aweq_gran gran, int group, unsigned char *codes, float *step, int *zp,
                                          float *epsmu, const BiasIO &bias, void *ws, size_t ws_bytes,
                                          aweq_dev_status *st, void *stream)
{
    aweq_status rc = check_matrix(W, dt, C_out, C_in, ldw, false);
    if (rc != AWEQ_OK) return rc;
    rc = check_quant(bits, gran, group, C_in);
    if (rc != AWEQ_OK) return rc;
    if (!codes || !step || !zp) return AWEQ_ERR_NULL;
    if (!aligned(codes, 16) || (s && !aligned(s, 16)) || (mu_hat && !aligned(mu_hat, 16))) return AWEQ_ERR_ALIGN;
    rc = check_ws(ws, ws_bytes, eq_ws_bytes(C_out, C_in, bits, gran, group));
    if (rc != AWEQ_OK) return rc;
    AWEQ_LOGF("aweq_equalize_quantize C_out=%lld C_in=%lld bits=%d gran=%d group=%d bytes=%lld\n", C_out, C_in, bits,
              (int)gran, group, 2 * C_out * C_in + C_out * C_in * bits / 8);
    cudaStream_t cs = (cudaStream_t)stream;
    if (gran == AWEQ_PER_ROW) {
        if (!rowquant_supported(C_out, C_in)) return AWEQ_ERR_SHAPE;
        return run_rowquant(W, dt, C_out, C_in, ldw, s, mu_hat, bits, true, codes, step, zp, epsmu, bias, st, cs);
    }
    if (gran == AWEQ_PER_GROUP && groupquant_supported(bits, group))
        return run_groupquant(W, dt, C_out, C_in, ldw, s, mu_hat, bits, codes, step, zp, epsmu, bias, ws, cs);
    if (gran == AWEQ_PER_GROUP)
        return run_warpquant(W, dt, C_out, C_in, ldw, s, mu_hat, bits, true, group, nullptr, codes, step, zp, epsmu,
                             bias, st, cs);
    // per tensor: column extremes of W -> extremes of diag(s) W -> static-range quantiser
    char *base = reinterpret_cast<char *>(ws);
    float *cmin = reinterpret_cast<float *>(base);
    float *cmax = cmin + C_in;
    float *lo_hi = reinterpret_cast<float *>(base + round256((size_t)C_in * 8));
    void *ws2 = base + round256((size_t)C_in * 8) + 256;
    rc = run_wrange(W, dt, C_out, C_in, ldw, cmin, cmax, 0, ws2, st, cs);
    if (rc != AWEQ_OK) return rc;
    rc = run_scaled_tensor_range(cmin, cmax, s, C_in, lo_hi, cs);
    if (rc != AWEQ_OK) return rc;
    return run_warpquant(W, dt, C_out, C_in, ldw, s, mu_hat, bits, true, 0, lo_hi, codes, step, zp, epsmu, bias, st,
                         cs);
}

aweq_status aweq_equalize_quantize(const void *W, aweq_dtype dt, long long C_out, long long C_in, long long ldw,
                                   const float *s, const float *mu_hat, int bits, aweq_gran gran, int group,
                                   unsigned char *codes, float *step, int *zp, float *epsmu, void *ws,
                                   size_t ws_bytes, aweq_dev_status *st, void *stream)
{
    const BiasIO none = {nullptr, nullptr, nullptr, 0};
    return equalize_quantize_impl(W, dt, C_out, C_in, ldw, s, mu_hat, bits, gran, group, codes, step, zp, epsmu, none,
                                  ws, ws_bytes, st, stream);
}

aweq_status aweq_bias_correct(const float *epsmu, const void *W, aweq_dtype dt, const float *s,
                              const unsigned char *codes, const float *step, const int *zp, const float *mu_hat,
                              long long C_out, long long C_in, long long ldw, int bits, aweq_gran gran, int group,
                              const void *bias_in, void *bias_out, float *bias_out_f32, aweq_dtype bias_dt,
                              aweq_dev_status *st, void *stream)
{
    (void)st;
    if (C_out <= 0) return AWEQ_ERR_SHAPE;
    if (!bias_out && !bias_out_f32) return AWEQ_ERR_NULL;
    if (bias_dt != AWEQ_F16 && bias_dt != AWEQ_BF16) return AWEQ_ERR_DTYPE;
    if (epsmu) return run_bias_apply(epsmu, bias_in, bias_out, bias_out_f32, bias_dt, C_out, (cudaStream_t)stream);
    aweq_status rc = check_matrix(W, dt, C_out, C_in, ldw, false);
    if (rc != AWEQ_OK) return rc;
    rc = check_quant(bits, gran, group, C_in);
    if (rc != AWEQ_OK) return rc;
    if (!codes || !step || !zp || !mu_hat) return AWEQ_ERR_NULL;
    return run_bias_gemv(W, dt, C_out, C_in, ldw, s, codes, step, zp, mu_hat, bits, gran, group, bias_in, bias_out,
                         bias_out_f32, bias_dt, (cudaStream_t)stream);
}

aweq_status aweq_quant_act(const void *X, aweq_dtype dt, long long N, long long C_in, long long ldx,
                           const float *rinv, int bits, aweq_gran gran, const float *tensor_lo_hi,
                           unsigned char *Xq, float *step, int *zp, aweq_dev_status *st, void *stream)
{
    aweq_status rc = check_matrix(X, dt, N, C_in, ldx, false);
    if (rc != AWEQ_OK) return rc;
    if (bits < 2 || bits > 8) return AWEQ_ERR_BITS;
    if (!Xq || !step || !zp) return AWEQ_ERR_NULL;
    if (!aligned(Xq, 16) || (rinv && !aligned(rinv, 16))) return AWEQ_ERR_ALIGN;
    AWEQ_LOGF("aweq_quant_act N=%lld C_in=%lld bits=%d gran=%d bytes=%lld\n", N, C_in, bits, (int)gran, 3 * N * C_in + 8 * N);
    cudaStream_t cs = (cudaStream_t)stream;
    if (gran == AWEQ_PER_ROW) {
        if (!rowquant_supported(N, C_in)) return AWEQ_ERR_SHAPE;
        const BiasIO none = {nullptr, nullptr, nullptr, 0};
        return run_rowquant(X, dt, N, C_in, ldx, rinv, nullptr, bits, false, Xq, step, zp, nullptr, none, st, cs);
    }
    if (gran == AWEQ_PER_TENSOR) {
        if (!tensor_lo_hi) return AWEQ_ERR_NULL;
        const BiasIO none = {nullptr, nullptr, nullptr, 0};
        return run_warpquant(X, dt, N, C_in, ldx, rinv, nullptr, bits, false, 0, tensor_lo_hi, Xq, step, zp, nullptr,
                             none, st, cs);
    }
    return AWEQ_ERR_UNSUPPORTED;
}

// ------------------------------------------------------------------ layer pass
// workspace layout: [column-reduction scratch | scratch of step 4]
static size_t layer_ws_parts(const aweq_layer_args *a, size_t *col_part)
{
    size_t col = stats_wrange_fusable(a->N, a->C_in, a->C_out, a->n_w) ? colreduce_fused_ws_bytes(a->N, a->C_in)
                                                     : colreduce_ws_bytes(a->N, a->C_in);
    size_t eq = 0;
    for (int i = 0; i < a->n_w; ++i) {
        size_t c = colreduce_ws_bytes(a->C_out[i], a->C_in);
        if (c > col) col = c;
        size_t e = eq_ws_bytes(a->C_out[i], a->C_in, a->bits, a->gran, a->group);
        if (e > eq) eq = e;
    }
    col = round256(col);
    if (col_part) *col_part = col;
    return col + round256(eq);
}

int aweq_layer_pass_fuses_ranges(const aweq_layer_args *args)
{
    return args && args->C_out && stats_wrange_fusable(args->N, args->C_in, args->C_out, args->n_w) ? 1 : 0;
}

size_t aweq_layer_pass_workspace_bytes(const aweq_layer_args *args)
{
    if (!args || args->n_w <= 0 || !args->C_out || args->C_in <= 0) return 0;
    return layer_ws_parts(args, nullptr);
}

// A profiling hook.  While the stream is being captured into a CUDA graph an ordinary record would
// only become an edge of the graph; as an external record it becomes a node of its own, so the
// event is recorded anew on every replay and can be read back afterwards.
static cudaError_t record_hook(void *ev, cudaStream_t cs)
{
    cudaStreamCaptureStatus cap = cudaStreamCaptureStatusNone;
    cudaError_t e = cudaStreamIsCapturing(cs, &cap);
    if (e != cudaSuccess) return e;
    return cudaEventRecordWithFlags((cudaEvent_t)ev, cs,
                                    cap == cudaStreamCaptureStatusActive ? cudaEventRecordExternal : cudaEventRecordDefault);
}

aweq_status aweq_layer_pass(const aweq_layer_args *a, void *ws, size_t ws_bytes, aweq_dev_status *st, void *stream)
{
    if (!a) return AWEQ_ERR_NULL;
    if (a->n_w <= 0 || !a->W || !a->C_out || !a->ldw || !a->codes || !a->step || !a->zp) return AWEQ_ERR_NULL;
    if (!a->xmin || !a->xmax || !a->xmean || !a->wmin || !a->wmax || !a->s || !a->rinv || !a->mu_hat)
        return AWEQ_ERR_NULL;
    aweq_status rc = check_matrix(a->X, a->dt, a->N, a->C_in, a->ldx, false);
    if (rc != AWEQ_OK) return rc;
    rc = check_quant(a->bits, a->gran, a->group, a->C_in);
    if (rc != AWEQ_OK) return rc;
    for (int i = 0; i < a->n_w; ++i) {
        rc = check_matrix(a->W[i], a->dt, a->C_out[i], a->C_in, a->ldw[i], false);
        if (rc != AWEQ_OK) return rc;
        if (!a->codes[i] || !a->step[i] || !a->zp[i]) return AWEQ_ERR_NULL;
    }
    const bool bc = !(a->flags & AWEQ_FLAG_NO_BIAS_CORRECT);
    if (bc && (!a->epsmu || (!a->bias_out && !a->bias_out_f32))) return AWEQ_ERR_NULL;
    for (int i = 0; bc && i < a->n_w; ++i) {
        if (!a->epsmu[i]) return AWEQ_ERR_NULL;
        if (!(a->bias_out && a->bias_out[i]) && !(a->bias_out_f32 && a->bias_out_f32[i])) return AWEQ_ERR_NULL;
    }
    if (a->Xq && (!a->act_step || !a->act_zp)) return AWEQ_ERR_NULL;
    if ((a->stat_negmin_max == nullptr) != (a->stat_sum_count == nullptr)) return AWEQ_ERR_NULL;
    if ((a->flags & AWEQ_FLAG_MERGED_STATS) && !a->stat_negmin_max) return AWEQ_ERR_NULL;
    if (a->stat_negmin_max && (!aligned(a->stat_negmin_max, 4) || !aligned(a->stat_sum_count, 8))) return AWEQ_ERR_ALIGN;
    size_t col_part = 0;
    const size_t need = layer_ws_parts(a, &col_part);
    rc = check_ws(ws, ws_bytes, need);
    if (rc != AWEQ_OK) return rc;
    char *base = reinterpret_cast<char *>(ws);
    void *ws_col = base;
    void *ws_eq = base + col_part;
    const size_t ws_eq_bytes = need - col_part;

    cudaStream_t cs = (cudaStream_t)stream;
    const int kAllPhases = AWEQ_FLAG_PHASE_REDUCE | AWEQ_FLAG_PHASE_QUANT | AWEQ_FLAG_PHASE_ACT;
    const int phases = (a->flags & kAllPhases) ? (a->flags & kAllPhases) : kAllPhases;
    // steps 1-2
    if (phases & AWEQ_FLAG_PHASE_REDUCE) {
        if (a->ev_stats_begin) AWEQ_CUDA_OK(record_hook(a->ev_stats_begin, cs));
        if (!aligned(a->xmin, 16) || !aligned(a->xmax, 16) || !aligned(a->xmean, 4)) return AWEQ_ERR_ALIGN;
        if (stats_wrange_fusable(a->N, a->C_in, a->C_out, a->n_w)) {
            // steps 1 and 2 in one launch: every CTA of the sweep also takes its share of the rows of the
            // matrices this input feeds (they have the same columns), so step 2 has no launch, fill or
            // drain of its own.  The hook interval then covers both steps.
            AWEQ_LOGF("aweq_stats + aweq_wrange x%d N=%lld C_in=%lld bytes=%lld (one launch)\n", a->n_w, a->N, a->C_in,
                      2 * a->N * a->C_in);
            rc = run_stats_wrange(a->X, a->dt, a->N, a->C_in, a->ldx, a->xmin, a->xmax, a->xmean, a->W, a->C_out, a->ldw,
                                  a->n_w, a->wmin, a->wmax, ws_col, st, cs, a->stat_negmin_max, a->stat_sum_count);
            if (rc != AWEQ_OK) return rc;
            if (a->ev_stats_end) AWEQ_CUDA_OK(record_hook(a->ev_stats_end, cs));
        } else {
            if (a->stat_negmin_max) {
                // the sweep that also leaves the exchange form of the statistics
                AWEQ_LOGF("aweq_stats N=%lld C_in=%lld (with exchange buffers) bytes=%lld\n", a->N, a->C_in, 2 * a->N * a->C_in);
                rc = run_stats(a->X, a->dt, a->N, a->C_in, a->ldx, a->xmin, a->xmax, a->xmean, nullptr, nullptr, 0, ws_col,
                               st, cs, a->stat_negmin_max, a->stat_sum_count);
            } else {
                rc = aweq_stats(a->X, a->dt, a->N, a->C_in, a->ldx, a->xmin, a->xmax, a->xmean, nullptr, nullptr, 0, ws_col,
                                col_part, st, stream);
            }
            if (rc != AWEQ_OK) return rc;
            if (a->ev_stats_end) AWEQ_CUDA_OK(record_hook(a->ev_stats_end, cs));
            // step 2: the matrices share the input, hence one range per input channel over all of them
            AWEQ_LOGF("aweq_wrange x%d C_in=%lld\n", a->n_w, a->C_in);
            rc = run_wrange_multi(a->W, a->C_out, a->ldw, a->n_w, a->dt, a->C_in, a->wmin, a->wmax, 0, ws_col, st, cs);
            if (rc != AWEQ_OK) return rc;
        }
    }
    const bool eq = !(a->flags & AWEQ_FLAG_NO_EQUALIZE);
    // without equalisation the layer sees x itself, so E[x^] = E[x]
    const float *s_used = eq ? a->s : nullptr;
    const float *rinv_used = eq ? a->rinv : nullptr;
    const float *mu_used = eq ? a->mu_hat : a->xmean;
    if (phases & AWEQ_FLAG_PHASE_QUANT) {
    if (a->flags & AWEQ_FLAG_MERGED_STATS) {
        rc = run_stats_from_exchange(a->stat_negmin_max, a->stat_sum_count, a->C_in, a->xmin, a->xmax, a->xmean, cs);
        if (rc != AWEQ_OK) return rc;
    }
    // step 3
    rc = ((a->flags & AWEQ_FLAG_ABSMAX_CRITERION) ? aweq_factors_absmax : aweq_factors)(
        a->xmin, a->xmax, a->xmean, a->wmin, a->wmax, a->C_in, a->s, a->rinv, a->mu_hat, a->pX, a->pW, a->scalars, st,
        stream);
    if (rc != AWEQ_OK) return rc;
    // steps 4-5 per matrix: the corrected bias is written by the quantiser itself
    for (int i = 0; i < a->n_w; ++i) {
        float *em = bc ? a->epsmu[i] : nullptr;
        BiasIO bias = {nullptr, nullptr, nullptr, a->dt == AWEQ_BF16};
        if (bc) {
            bias.in = reinterpret_cast<const uint16_t *>(a->bias_in ? a->bias_in[i] : nullptr);
            bias.out = reinterpret_cast<uint16_t *>(a->bias_out ? a->bias_out[i] : nullptr);
            bias.out_f32 = a->bias_out_f32 ? a->bias_out_f32[i] : nullptr;
        }
        rc = equalize_quantize_impl(a->W[i], a->dt, a->C_out[i], a->C_in, a->ldw[i], s_used, bc ? mu_used : nullptr,
                                    a->bits, a->gran, a->group, a->codes[i], a->step[i], a->zp[i], em, bias, ws_eq,
                                    ws_eq_bytes, st, stream);
        if (rc != AWEQ_OK) return rc;
    }
    }
    // step 6
    if (a->Xq && (phases & AWEQ_FLAG_PHASE_ACT)) {
        if (a->ev_act_begin) AWEQ_CUDA_OK(record_hook(a->ev_act_begin, cs));
        rc = aweq_quant_act(a->X, a->dt, a->N, a->C_in, a->ldx, rinv_used, a->act_bits ? a->act_bits : 8, AWEQ_PER_ROW,
                            nullptr, a->Xq, a->act_step, a->act_zp, st, stream);
        if (rc != AWEQ_OK) return rc;
        if (a->ev_act_end) AWEQ_CUDA_OK(record_hook(a->ev_act_end, cs));
    }
    return AWEQ_OK;
}

// ------------------------------------------------------------------ folding 1/s into the producer
aweq_status aweq_fold_scale(const void *P, aweq_dtype dt, long long rows, long long cols, long long ld,
                            const float *rinv, void *out, long long ld_out, void *stream)
{
    if (!P || !rinv || !out) return AWEQ_ERR_NULL;
    if (dt != AWEQ_F16 && dt != AWEQ_BF16) return AWEQ_ERR_DTYPE;
    if (rows <= 0 || cols <= 0 || rows > (1ll << 40) || cols > (1ll << 30)) return AWEQ_ERR_SHAPE;
    if (ld < cols || ld_out < cols) return AWEQ_ERR_ALIGN;
    if (!aligned(P, 2) || !aligned(out, 2) || !aligned(rinv, 4)) return AWEQ_ERR_ALIGN;
    AWEQ_LOGF("aweq_fold_scale rows=%lld cols=%lld bytes=%lld\n", rows, cols, 4 * rows * cols + 4 * rows);
    return run_fold_scale(P, dt, rows, cols, ld, rinv, out, ld_out, (cudaStream_t)stream);
}

// ------------------------------------------------------------------ signed relabelling
aweq_status aweq_relabel_signed(const unsigned char *codes, long long n, signed char *out, const int *zp, long long nz,
                                int *zp_out, void *stream)
{
    if (!codes || !out) return AWEQ_ERR_NULL;
    if ((zp == nullptr) != (zp_out == nullptr)) return AWEQ_ERR_NULL;
    if (n <= 0 || nz < 0 || (zp && nz == 0)) return AWEQ_ERR_SHAPE;
    return run_relabel_signed(codes, n, out, zp, zp ? nz : 0, zp_out, (cudaStream_t)stream);
}

// ------------------------------------------------------------------ forward check
size_t aweq_forward_check_workspace_bytes(long long N, long long C_in, long long C_out)
{
    if (N <= 0 || C_in <= 0 || C_out <= 0) return 0;
    return forward_check_ws_bytes(N, C_in, C_out);
}

aweq_status aweq_forward_check(const unsigned char *Xq, const float *act_step, const int *act_zp,
                               const unsigned char *Wq, const float *w_step, const int *w_zp, const float *bias_q,
                               const void *X, const void *W, aweq_dtype dt, const void *bias, long long N,
                               long long C_in, long long C_out, double *mean_err, double *sums, void *ws,
                               size_t ws_bytes, void *stream)
{
    if (!Xq || !act_step || !act_zp || !Wq || !w_step || !w_zp || !X || !W || !mean_err || !sums) return AWEQ_ERR_NULL;
    if (dt != AWEQ_F16 && dt != AWEQ_BF16) return AWEQ_ERR_DTYPE;
    if (N <= 0 || C_in <= 0 || C_out <= 0 || C_in % 16 || C_out % 8) return AWEQ_ERR_SHAPE;
    if (C_in > (1ll << 30) || C_out > (1ll << 30) || N > (1ll << 34)) return AWEQ_ERR_SHAPE;
    if (!aligned(Xq, 16) || !aligned(Wq, 16) || !aligned(X, 16) || !aligned(W, 16)) return AWEQ_ERR_ALIGN;
    if (!ws || !aligned(ws, 256) || ws_bytes < forward_check_ws_bytes(N, C_in, C_out)) return AWEQ_ERR_WORKSPACE;
    AWEQ_LOGF("aweq_forward_check N=%lld C_in=%lld C_out=%lld flops=%.3e\n", N, C_in, C_out, 4.0 * N * C_in * C_out);
    return run_forward_check(Xq, act_step, act_zp, Wq, w_step, w_zp, bias_q, X, W, dt, bias, N, C_in, C_out, mean_err,
                             sums, ws, ws_bytes, (cudaStream_t)stream);
}

size_t aweq_forward_check_weights_workspace_bytes(long long N, long long C_in, long long C_out)
{
    if (N <= 0 || C_in <= 0 || C_out <= 0) return 0;
    return forward_check_weights_ws_bytes(N, C_in, C_out);
}

aweq_status aweq_forward_check_weights(const unsigned char *codes, const float *step, const int *zp, int bits,
                                       aweq_gran gran, int group, const float *rinv, const float *bias_q,
                                       const void *X, const void *W, aweq_dtype dt, const void *bias, long long N,
                                       long long C_in, long long C_out, double *mean_err, double *sums, void *ws,
                                       size_t ws_bytes, void *stream)
{
    if (!codes || !step || !zp || !X || !W || !mean_err || !sums) return AWEQ_ERR_NULL;
    if (dt != AWEQ_F16 && dt != AWEQ_BF16) return AWEQ_ERR_DTYPE;
    if (N <= 0 || C_in <= 0 || C_out <= 0 || C_in % 16 || C_out % 8) return AWEQ_ERR_SHAPE;
    if (C_in > (1ll << 30) || C_out > (1ll << 30) || N > (1ll << 34)) return AWEQ_ERR_SHAPE;
    aweq_status rc = check_quant(bits, gran, group, C_in);
    if (rc != AWEQ_OK) return rc;
    if (!aligned(X, 16) || !aligned(W, 16) || (rinv && !aligned(rinv, 16))) return AWEQ_ERR_ALIGN;
    if (!ws || !aligned(ws, 256) || ws_bytes < forward_check_weights_ws_bytes(N, C_in, C_out)) return AWEQ_ERR_WORKSPACE;
    AWEQ_LOGF("aweq_forward_check_weights N=%lld C_in=%lld C_out=%lld bits=%d flops=%.3e\n", N, C_in, C_out, bits,
              4.0 * N * C_in * C_out);
    return run_forward_check_weights(codes, step, zp, bits, gran, group, rinv, bias_q, X, W, dt, bias, N, C_in, C_out,
                                     mean_err, sums, ws, ws_bytes, (cudaStream_t)stream);
}

// ------------------------------------------------------------------ running a calibrated layer
static aweq_status check_codes(const void *Q, long long cols, long long ld)
{
    if (cols <= 0 || cols % 16 || cols > AWEQ_LINEAR_MAX_C_IN) return AWEQ_ERR_SHAPE;
    if (!aligned(Q, 16) || ld < cols || ld % 16 || ld > (1ll << 40)) return AWEQ_ERR_ALIGN;
    return AWEQ_OK;
}

aweq_status aweq_code_sums(const unsigned char *codes, long long rows, long long cols, long long ld, int *sums, void *stream)
{
    if (!codes || !sums) return AWEQ_ERR_NULL;
    if (rows <= 0 || rows > (1ll << 30)) return AWEQ_ERR_SHAPE;
    aweq_status rc = check_codes(codes, cols, ld);
    if (rc != AWEQ_OK) return rc;
    AWEQ_LOGF("aweq_code_sums rows=%lld cols=%lld bytes=%lld\n", rows, cols, rows * cols);
    return run_code_sums(codes, rows, cols, ld, sums, (cudaStream_t)stream);
}

aweq_status aweq_linear_w8a8(const unsigned char *Xq, long long ldx, const float *act_step, const int *act_zp,
                             aweq_gran act_gran, const unsigned char *Wq, long long ldw, const float *w_step,
                             const int *w_zp, const int *w_sum, aweq_gran w_gran, const float *bias, long long N,
                             long long C_in, long long C_out, void *out, aweq_dtype dt, long long ldo,
                             aweq_dev_status *st, void *stream)
{
    if (dt != AWEQ_F16 && dt != AWEQ_BF16) return AWEQ_ERR_DTYPE;
    if ((act_gran != AWEQ_PER_ROW && act_gran != AWEQ_PER_TENSOR) || (w_gran != AWEQ_PER_ROW && w_gran != AWEQ_PER_TENSOR))
        return AWEQ_ERR_UNSUPPORTED;
    if (N < 0 || N > 0x7fffffffll || C_out <= 0 || C_out > (1ll << 30)) return AWEQ_ERR_SHAPE;
    if (!Wq || !w_step || !w_zp || !w_sum) return AWEQ_ERR_NULL;
    if (N > 0 && (!Xq || !act_step || !act_zp || !out)) return AWEQ_ERR_NULL;
    aweq_status rc = check_codes(Wq, C_in, ldw);
    if (rc == AWEQ_OK) rc = check_codes(Xq, C_in, ldx);
    if (rc != AWEQ_OK) return rc;
    if (!aligned(out, 2) || ldo < C_out || !aligned(act_step, 4) || !aligned(act_zp, 4) || !aligned(w_step, 4) ||
        !aligned(w_zp, 4) || !aligned(w_sum, 4) || (bias && !aligned(bias, 4)))
        return AWEQ_ERR_ALIGN;
    if (N == 0) return AWEQ_OK;
    AWEQ_LOGF("aweq_linear_w8a8 N=%lld C_in=%lld C_out=%lld ops=%.3e\n", N, C_in, C_out, 2.0 * N * C_in * C_out);
    Linear8Args a = {};
    a.X = Xq; a.W = Wq; a.ldx = ldx; a.ldw = ldw; a.ldo = ldo; a.N = N;
    a.x_step = act_step; a.w_step = w_step; a.bias = bias; a.x_zp = act_zp; a.w_zp = w_zp; a.w_sum = w_sum;
    a.x_inc = act_gran == AWEQ_PER_ROW; a.w_inc = w_gran == AWEQ_PER_ROW;
    a.K = (int)C_in; a.O = (int)C_out; a.out = reinterpret_cast<uint16_t *>(out); a.st = st;
    return run_linear8(a, dt, (cudaStream_t)stream);
}

static aweq_status check_mx4(int fmt, long long rows, long long cols)
{
    if (fmt != AWEQ_MX4_E8M0 && fmt != AWEQ_MX4_E4M3) return AWEQ_ERR_UNSUPPORTED;
    if (rows < 0 || rows > 0x7fffffffll || cols <= 0 || cols % 32 || cols > AWEQ_LINEAR_MAX_C_IN) return AWEQ_ERR_SHAPE;
    if ((rows + 127) / 128 * mx4_row_tiles(cols, fmt) > 0x7fffffffll) return AWEQ_ERR_SHAPE;
    return AWEQ_OK;
}

size_t aweq_mx4_scale_bytes(long long rows, long long cols, aweq_mx4_format fmt)
{
    if (check_mx4(fmt, rows, cols) != AWEQ_OK) return 0;
    return (size_t)((rows + 127) / 128 * mx4_row_tiles(cols, fmt)) * kMx4Tile;
}

aweq_status aweq_quant_mx4(const void *X, aweq_dtype dt, long long rows, long long cols, long long ld, const float *scale,
                           aweq_mx4_format fmt, unsigned char *codes, unsigned char *scales, float *row_step, const float *mu,
                           float *epsmu, aweq_dev_status *st, void *stream)
{
    if (dt != AWEQ_F16 && dt != AWEQ_BF16) return AWEQ_ERR_DTYPE;
    aweq_status rc = check_mx4(fmt, rows, cols);
    if (rc != AWEQ_OK) return rc;
    if ((mu == nullptr) != (epsmu == nullptr)) return AWEQ_ERR_NULL;
    if (rows == 0) return AWEQ_OK;
    if (!X || !codes || !scales || (fmt == AWEQ_MX4_E4M3 && !row_step)) return AWEQ_ERR_NULL;
    if (!aligned(X, 16) || ld < cols || ld % 8 || !aligned(codes, 16) || !aligned(scales, 16) || !aligned(scale, 16) || !aligned(mu, 16) ||
        !aligned(row_step, 4) || !aligned(epsmu, 4))
        return AWEQ_ERR_ALIGN;
    AWEQ_LOGF("aweq_quant_mx4 rows=%lld cols=%lld fmt=%d bytes=%lld\n", rows, cols, (int)fmt, rows * cols * 5 / 2);
    return run_quant_mx4(X, dt, rows, cols, ld, scale, fmt, codes, scales, row_step, mu, epsmu, st, (cudaStream_t)stream);
}

aweq_status aweq_dequant_mx4(const unsigned char *codes, const unsigned char *scales, const float *row_step, aweq_mx4_format fmt,
                             long long rows, long long cols, void *out, aweq_dtype dt, long long ldo, void *stream)
{
    if (dt != AWEQ_F16 && dt != AWEQ_BF16) return AWEQ_ERR_DTYPE;
    aweq_status rc = check_mx4(fmt, rows, cols);
    if (rc != AWEQ_OK || rows == 0) return rc;
    if (!out || !codes || !scales || (fmt == AWEQ_MX4_E4M3 && !row_step)) return AWEQ_ERR_NULL;
    if (!aligned(out, 16) || ldo < cols || ldo % 8 || !aligned(codes, 16) || !aligned(scales, 16) || !aligned(row_step, 4)) return AWEQ_ERR_ALIGN;
    return run_dequant_mx4(codes, scales, row_step, fmt, rows, cols, out, dt, ldo, (cudaStream_t)stream);
}

aweq_status aweq_linear_mx4(const unsigned char *Xq, const unsigned char *x_scales, const float *x_step, const unsigned char *Wq,
                            const unsigned char *w_scales, const float *w_step, aweq_mx4_format fmt, const float *bias, long long N,
                            long long C_in, long long C_out, void *out, aweq_dtype dt, long long ldo, aweq_dev_status *st, void *stream)
{
    if (dt != AWEQ_F16 && dt != AWEQ_BF16) return AWEQ_ERR_DTYPE;
    aweq_status rc = check_mx4(fmt, N, C_in);
    if (rc == AWEQ_OK) rc = check_mx4(fmt, C_out, C_in);
    if (rc != AWEQ_OK) return rc;
    if (C_out <= 0 || C_out > (1ll << 30)) return AWEQ_ERR_SHAPE;
    const bool steps = fmt == AWEQ_MX4_E4M3;
    if (!Wq || !w_scales || (steps && !w_step)) return AWEQ_ERR_NULL;
    if (N > 0 && (!Xq || !x_scales || !out || (steps && !x_step))) return AWEQ_ERR_NULL;
    if (!aligned(Xq, 16) || !aligned(Wq, 16) || !aligned(x_scales, 16) || !aligned(w_scales, 16) || !aligned(x_step, 4) || !aligned(w_step, 4) ||
        !aligned(bias, 4) || !aligned(out, 2) || ldo < C_out)
        return AWEQ_ERR_ALIGN;
    if (N == 0) return AWEQ_OK;
    AWEQ_LOGF("aweq_linear_mx4 N=%lld C_in=%lld C_out=%lld fmt=%d ops=%.3e\n", N, C_in, C_out, (int)fmt, 2.0 * N * C_in * C_out);
    Mx4LinearArgs a = {};
    a.X = Xq; a.W = Wq; a.x_scales = x_scales; a.w_scales = w_scales; a.bias = bias; a.N = N; a.ldo = ldo;
    a.x_step = steps ? x_step : nullptr; a.w_step = steps ? w_step : nullptr;
    a.K = (int)C_in; a.O = (int)C_out; a.fmt = fmt; a.out = reinterpret_cast<uint16_t *>(out); a.st = st;
    return run_linear_mx4(a, dt, (cudaStream_t)stream);
}

aweq_status aweq_rope_table(const aweq_rope *r, long long n_pos, float *table, void *stream)
{
    if (!r || !table) return AWEQ_ERR_NULL;
    if (r->rotary_dim < 2 || r->rotary_dim > 256 || r->rotary_dim % 2 || n_pos <= 0 || n_pos > (1ll << 31)) return AWEQ_ERR_SHAPE;
    if (r->scaling < AWEQ_ROPE_NONE || r->scaling > AWEQ_ROPE_BANDS) return AWEQ_ERR_UNSUPPORTED;
    if (!(r->theta > 0) || !(r->attention > 0) || (r->scaling != AWEQ_ROPE_NONE && !(r->factor > 0))) return AWEQ_ERR_UNSUPPORTED;
    if (r->scaling == AWEQ_ROPE_BASE && r->rotary_dim < 4) return AWEQ_ERR_SHAPE;
    if (r->scaling == AWEQ_ROPE_BANDS && !(r->original_len > 0 && r->low >= 0 && r->high > r->low)) return AWEQ_ERR_UNSUPPORTED;
    if (!aligned(table, 4)) return AWEQ_ERR_ALIGN;
    return run_rope_table(r, n_pos, table, (cudaStream_t)stream);
}

static aweq_status check_cache(const aweq_kv_cache *c, int most_dim)
{
    if (!c || !c->k || !c->v) return AWEQ_ERR_NULL;
    if (c->dt != AWEQ_F16 && c->dt != AWEQ_BF16) return AWEQ_ERR_DTYPE;
    if (c->page_size <= 0 || c->page_size > (1 << 20) || c->n_kv_heads <= 0 || c->n_kv_heads > 4096 || c->n_pages <= 0 ||
        c->n_pages > 0x7fffffffll || c->head_dim <= 0 || c->head_dim % 8 || c->head_dim > most_dim)
        return AWEQ_ERR_SHAPE;
    if (!aligned(c->k, 16) || !aligned(c->v, 16) || c->page_stride % 8 || c->token_stride % 8 || c->head_stride % 8 ||
        c->page_stride < 0 || c->token_stride < c->head_dim || c->head_stride < c->head_dim)
        return AWEQ_ERR_ALIGN;
    return AWEQ_OK;
}

static KvAppendArgs append_args(const aweq_kv_cache *cache, const void *k, long long ldk, const void *v, long long ldv, const int *pos,
                                long long n_tokens, const float *rope, long long n_pos, int rotary_dim, int interleaved, const void *q,
                                long long ldq, int n_heads, void *q_out, long long ld_qout, aweq_dev_status *st)
{
    KvAppendArgs a = {};
    a.ck = reinterpret_cast<uint16_t *>(cache->k); a.cv = reinterpret_cast<uint16_t *>(cache->v);
    a.n_pages = cache->n_pages; a.page_stride = cache->page_stride; a.token_stride = cache->token_stride;
    a.head_stride = cache->head_stride; a.page_size = cache->page_size; a.n_kv = cache->n_kv_heads;
    a.head_dim = cache->head_dim; a.k = reinterpret_cast<const uint16_t *>(k); a.v = reinterpret_cast<const uint16_t *>(v);
    a.q = reinterpret_cast<const uint16_t *>(q); a.q_out = reinterpret_cast<uint16_t *>(q_out);
    a.ldk = ldk; a.ldv = ldv; a.ldq = ldq; a.ld_qout = ld_qout; a.n_heads = q ? n_heads : 0; a.pos = pos; a.n_tokens = n_tokens;
    a.rope = rope; a.n_pos = n_pos; a.rd = rope ? rotary_dim : 0; a.interleaved = interleaved; a.st = st;
    return a;
}

aweq_status aweq_kv_append(const aweq_kv_cache *cache, const int *page_table, long long n_seq, long long pages_per_seq,
                           long long ld_table, const void *k, long long ldk, const void *v, long long ldv,
                           const int *pos, const int *seq, long long first, long long n_tokens, const float *rope,
                           long long n_pos, int rotary_dim, int interleaved, const void *q, long long ldq, int n_heads,
                           void *q_out, long long ld_qout, aweq_dev_status *st, void *stream)
{
    aweq_status rc = check_cache(cache, 256);
    if (rc != AWEQ_OK) return rc;
    const long long row = (long long)cache->n_kv_heads * cache->head_dim;
    if (n_tokens < 0 || n_tokens > 0x7fffffffll || n_seq <= 0 || n_seq > 0x7fffffffll || pages_per_seq <= 0 ||
        pages_per_seq > 0x7fffffffll || first < 0)
        return AWEQ_ERR_SHAPE;
    if (rope && (rotary_dim < 2 || rotary_dim % 2 || rotary_dim > cache->head_dim || n_pos <= 0)) return AWEQ_ERR_SHAPE;
    if ((q == nullptr) != (q_out == nullptr)) return AWEQ_ERR_NULL;
    if (q && (n_heads <= 0 || n_heads > 65536)) return AWEQ_ERR_SHAPE;
    if (!seq && n_tokens > n_seq) return AWEQ_ERR_SHAPE;
    if (n_tokens == 0) return AWEQ_OK;
    if (!page_table || !k || !v || !pos) return AWEQ_ERR_NULL;
    if (ld_table < pages_per_seq || ldk < row || ldv < row || !aligned(k, 2) || !aligned(v, 2) || !aligned(pos, 4) ||
        !aligned(seq, 4) || !aligned(page_table, 4) || !aligned(rope, 4))
        return AWEQ_ERR_ALIGN;
    if (q) {
        const long long qrow = (long long)n_heads * cache->head_dim;
        if (ldq < qrow || ld_qout < qrow || !aligned(q, 2) || !aligned(q_out, 2)) return AWEQ_ERR_ALIGN;
    }
    AWEQ_LOGF("aweq_kv_append tokens=%lld heads=%d kv_heads=%d head_dim=%d rotary_dim=%d bytes=%lld\n", n_tokens,
              q ? n_heads : 0, cache->n_kv_heads, cache->head_dim, rope ? rotary_dim : 0,
              n_tokens * ((q ? n_heads : 0) + 2 * cache->n_kv_heads) * cache->head_dim * 4);
    KvAppendArgs a = append_args(cache, k, ldk, v, ldv, pos, n_tokens, rope, n_pos, rotary_dim, interleaved, q, ldq, n_heads, q_out, ld_qout, st);
    a.page_table = page_table; a.n_seq = n_seq; a.pages_per_seq = pages_per_seq; a.ld_table = ld_table; a.seq = seq; a.first = first;
    return run_kv_append(a, cache->dt, (cudaStream_t)stream);
}

aweq_status aweq_kv_append_slots(const aweq_kv_cache *cache, const long long *slot, const void *k, long long ldk, const void *v,
                                 long long ldv, const int *pos, long long n_tokens, const float *rope, long long n_pos, int rotary_dim,
                                 int interleaved, const void *q, long long ldq, int n_heads, void *q_out, long long ld_qout,
                                 aweq_dev_status *st, void *stream)
{
    aweq_status rc = check_cache(cache, 256);
    if (rc != AWEQ_OK) return rc;
    const long long row = (long long)cache->n_kv_heads * cache->head_dim;
    if (n_tokens < 0 || n_tokens > 0x7fffffffll) return AWEQ_ERR_SHAPE;
    if (rope && (rotary_dim < 2 || rotary_dim % 2 || rotary_dim > cache->head_dim || n_pos <= 0)) return AWEQ_ERR_SHAPE;
    if ((q == nullptr) != (q_out == nullptr)) return AWEQ_ERR_NULL;
    if (q && (n_heads <= 0 || n_heads > 65536)) return AWEQ_ERR_SHAPE;
    if (n_tokens == 0) return AWEQ_OK;
    if (!slot || !k || !v || !pos) return AWEQ_ERR_NULL;
    if (ldk < row || ldv < row || !aligned(k, 2) || !aligned(v, 2) || !aligned(pos, 4) || !aligned(slot, 8) || !aligned(rope, 4)) return AWEQ_ERR_ALIGN;
    if (q) {
        const long long qrow = (long long)n_heads * cache->head_dim;
        if (ldq < qrow || ld_qout < qrow || !aligned(q, 2) || !aligned(q_out, 2)) return AWEQ_ERR_ALIGN;
    }
    KvAppendArgs a = append_args(cache, k, ldk, v, ldv, pos, n_tokens, rope, n_pos, rotary_dim, interleaved, q, ldq, n_heads, q_out, ld_qout, st);
    a.slot = slot;
    return run_kv_append(a, cache->dt, (cudaStream_t)stream);
}

constexpr long long kMostPages = 1ll << 22, kMostPlanned = 1ll << 30;        // (32-bit loops over the sequences step beyond the last)

size_t aweq_kv_plan_workspace_bytes(long long n_seq)
{
    return n_seq < 0 || n_seq > kMostPlanned ? 0 : kv_plan_ws_bytes(n_seq);
}

aweq_status aweq_kv_plan(int *page_table, long long n_seq, long long pages_per_seq, long long ld_table, int page_size, int *ring,
                         long long *state, long long n_pages, const int *held, const int *change, long long first,
                         long long max_tokens, int *own_len, int *start, int *seq, int *pos, long long *slot, const int *parent,
                         long long *mask, int words, void *ws, size_t ws_bytes, aweq_dev_status *st, void *stream)
{
    if (n_seq <= 0 || n_seq > kMostPlanned || pages_per_seq <= 0 || pages_per_seq > 0x7fffffffll || page_size <= 0 || page_size > (1 << 20) ||
        n_pages <= 0 || n_pages > kMostPages || max_tokens < 0 || max_tokens > 0x7fffffffll - 2048 || first < 0)
        return AWEQ_ERR_SHAPE;
    if (first + (double)pages_per_seq * page_size > 2147483647.0) return AWEQ_ERR_SHAPE;
    if (!page_table || !ring || !state || !held || !change || !own_len || !start) return AWEQ_ERR_NULL;
    if (max_tokens && (!seq || !pos || !slot)) return AWEQ_ERR_NULL;
    if ((parent == nullptr) != (mask == nullptr)) return AWEQ_ERR_NULL;
    if (parent && (words < 1 || words > kPlanMaxWords)) return AWEQ_ERR_SHAPE;
    if (ld_table < pages_per_seq || !aligned(page_table, 4) || !aligned(ring, 4) || !aligned(state, 8) || !aligned(held, 4) || !aligned(change, 4) ||
        !aligned(own_len, 4) || !aligned(start, 4) || !aligned(parent, 4) || own_len == held || own_len == change)
        return AWEQ_ERR_ALIGN;
    if (max_tokens && (!aligned(seq, 16) || !aligned(pos, 16) || !aligned(slot, 16) || !aligned(mask, 16))) return AWEQ_ERR_ALIGN;
    aweq_status rc = check_ws(ws, ws_bytes, kv_plan_ws_bytes(n_seq));
    if (rc != AWEQ_OK) return rc;
    AWEQ_LOGF("aweq_kv_plan seqs=%lld tokens=%lld page=%d words=%d\n", n_seq, max_tokens, page_size, parent ? words : 0);
    KvPlanArgs a = {};
    a.page_table = page_table; a.n_seq = n_seq; a.pages_per_seq = pages_per_seq; a.ld_table = ld_table; a.page_size = page_size;
    a.words = words; a.ring = ring; a.state = state; a.n_pages = n_pages; a.held = held; a.change = change; a.parent = parent;
    a.first = first; a.max_tokens = max_tokens; a.own_len = own_len; a.start = start; a.seq = seq; a.pos = pos; a.slot = slot;
    a.mask = mask; a.st = st;
    return run_kv_plan(a, ws, (cudaStream_t)stream);
}

aweq_status aweq_kv_accept(const aweq_kv_cache *cache, const int *page_table, long long n_seq, long long pages_per_seq,
                           long long ld_table, const int *base, const int *path, long long ld_path, int max_path, const int *n_path,
                           aweq_dev_status *st, void *stream)
{
    aweq_status rc = check_cache(cache, 256);
    if (rc != AWEQ_OK) return rc;
    const long long blocks = ((long long)cache->n_kv_heads * cache->head_dim / 4 + 127) / 128;
    if (n_seq < 0 || n_seq > 0x7fffffffll / blocks || pages_per_seq <= 0 || pages_per_seq > 0x7fffffffll || max_path < 0) return AWEQ_ERR_SHAPE;
    if (n_seq == 0 || max_path == 0) return AWEQ_OK;
    if (!page_table || !base || !path || !n_path) return AWEQ_ERR_NULL;
    if (ld_table < pages_per_seq || ld_path < max_path || !aligned(page_table, 4) || !aligned(base, 4) || !aligned(path, 4) || !aligned(n_path, 4))
        return AWEQ_ERR_ALIGN;
    KvAcceptArgs a = {};
    a.ck = reinterpret_cast<uint16_t *>(cache->k); a.cv = reinterpret_cast<uint16_t *>(cache->v);
    a.n_pages = cache->n_pages; a.page_stride = cache->page_stride; a.token_stride = cache->token_stride;
    a.head_stride = cache->head_stride; a.page_size = cache->page_size; a.n_kv = cache->n_kv_heads; a.head_dim = cache->head_dim;
    a.max_path = max_path; a.page_table = page_table; a.base = base; a.path = path; a.n_path = n_path; a.n_seq = n_seq;
    a.pages_per_seq = pages_per_seq; a.ld_table = ld_table; a.ld_path = ld_path; a.st = st;
    return run_kv_accept(a, (cudaStream_t)stream);
}

static aweq_status check_attention(const aweq_kv_cache *cache, long long prefix_len, long long max_own, long long n_seq, int n_q,
                                   int n_heads)
{
    aweq_status rc = check_cache(cache, 128);
    if (rc != AWEQ_OK) return rc;
    if (prefix_len < 0 || prefix_len > 0x7fffffffll || max_own < 0 || max_own > 0x7fffffffll || n_seq < 0 || n_q <= 0 ||
        n_heads <= 0 || n_heads % cache->n_kv_heads || n_heads > 65536 || n_q > 65536)
        return AWEQ_ERR_SHAPE;
    if (n_seq > 0x7fffffffll || (double)n_seq * n_q * n_heads > 2147483647.0) return AWEQ_ERR_SHAPE;
    return AWEQ_OK;
}

size_t aweq_prefix_attention_workspace_bytes(const aweq_kv_cache *cache, long long prefix_len, long long max_own, long long n_seq,
                                             int n_q, int n_heads)
{
    if (check_attention(cache, prefix_len, max_own, n_seq, n_q, n_heads) != AWEQ_OK || n_seq == 0) return 0;
    return prefix_attention_ws_bytes(cache, prefix_len, max_own, n_seq, n_q, n_heads);
}

aweq_status aweq_prefix_attention(const void *q, long long ldq, const aweq_kv_cache *cache, const int *prefix_pages,
                                  long long prefix_len, const int *page_table, long long pages_per_seq, long long ld_table,
                                  const int *own_len, long long max_own, long long n_seq, int n_q, int n_heads, float scale,
                                  void *out, long long ldo, void *ws, size_t ws_bytes, aweq_dev_status *st, void *stream)
{
    aweq_status rc = check_attention(cache, prefix_len, max_own, n_seq, n_q, n_heads);
    if (rc != AWEQ_OK) return rc;
    if (pages_per_seq < 0 || pages_per_seq > 0x7fffffffll) return AWEQ_ERR_SHAPE;
    if (n_seq == 0) return AWEQ_OK;
    if (!q || !out || !own_len || (prefix_len && !prefix_pages) || (max_own && pages_per_seq && !page_table)) return AWEQ_ERR_NULL;
    const long long row = (long long)n_heads * cache->head_dim;
    if (!aligned(q, 16) || !aligned(out, 16) || ldq < row || ldo < row || ldq % 8 || ldo % 8 || ld_table < pages_per_seq ||
        !aligned(prefix_pages, 4) || !aligned(page_table, 4) || !aligned(own_len, 4))
        return AWEQ_ERR_ALIGN;
    rc = check_ws(ws, ws_bytes, prefix_attention_ws_bytes(cache, prefix_len, max_own, n_seq, n_q, n_heads));
    if (rc != AWEQ_OK) return rc;
    AWEQ_LOGF("aweq_prefix_attention seqs=%lld n_q=%d heads=%d kv_heads=%d head_dim=%d prefix=%lld max_own=%lld\n", n_seq, n_q,
              n_heads, cache->n_kv_heads, cache->head_dim, prefix_len, max_own);
    AttentionArgs a = {};
    a.q = reinterpret_cast<const uint16_t *>(q); a.ck = reinterpret_cast<const uint16_t *>(cache->k);
    a.cv = reinterpret_cast<const uint16_t *>(cache->v); a.out = reinterpret_cast<uint16_t *>(out);
    a.ldq = ldq; a.ldo = ldo; a.n_pages = cache->n_pages; a.page_stride = cache->page_stride;
    a.token_stride = cache->token_stride; a.head_stride = cache->head_stride; a.page_size = cache->page_size;
    a.n_kv = cache->n_kv_heads; a.head_dim = cache->head_dim; a.n_heads = n_heads; a.n_q = n_q;
    a.prefix_pages = prefix_pages; a.page_table = page_table; a.own_len = own_len; a.prefix_len = prefix_len;
    a.pages_per_seq = pages_per_seq; a.ld_table = ld_table; a.max_own = max_own; a.n_seq = n_seq; a.scale = scale; a.st = st;
    return run_prefix_attention(a, cache, ws, (cudaStream_t)stream);
}

static aweq_status check_tree(const aweq_kv_cache *cache, long long prefix_len, long long max_own, long long n_seq, long long max_tokens,
                              int max_nodes, int n_heads)
{
    aweq_status rc = check_cache(cache, 128);
    if (rc != AWEQ_OK) return rc;
    if (prefix_len < 0 || prefix_len > 0x7fffffffll || max_own < 0 || max_own > 0x7fffffffll || n_seq < 0 || n_seq > (1ll << 24) || max_tokens < 0 ||
        max_tokens > 0x7fffffffll || max_nodes <= 0 || max_nodes > 64 * kPlanMaxWords || n_heads <= 0 || n_heads % cache->n_kv_heads || n_heads > 65536)
        return AWEQ_ERR_SHAPE;
    if ((double)max_tokens * n_heads > 2147483647.0 || (double)n_seq * 64 * kPlanMaxWords * n_heads > 2e12) return AWEQ_ERR_SHAPE;
    return AWEQ_OK;
}

size_t aweq_tree_attention_workspace_bytes(const aweq_kv_cache *cache, long long prefix_len, long long max_own, long long n_seq,
                                           long long max_tokens, int max_nodes, int n_heads)
{
    if (check_tree(cache, prefix_len, max_own, n_seq, max_tokens, max_nodes, n_heads) != AWEQ_OK || n_seq == 0 || max_tokens == 0) return 0;
    return tree_attention_ws_bytes(cache, prefix_len, max_own, n_seq, max_tokens, max_nodes, n_heads);
}

static aweq_status tree_attention(const void *q, long long ldq, const aweq_kv_cache *cache, const int *prefix_pages, long long prefix_len,
                                  const int *page_table, long long pages_per_seq, long long ld_table, const int *own_len, const int *start,
                                  const int *pos, long long first, const long long *mask, int words, long long max_own, long long n_seq,
                                  long long max_tokens, int max_nodes, int n_heads, float scale, void *out, long long ldo, void *ws,
                                  size_t ws_bytes, aweq_dev_status *st, void *stream)
{
    aweq_status rc = check_tree(cache, prefix_len, max_own, n_seq, max_tokens, max_nodes, n_heads);
    if (rc != AWEQ_OK) return rc;
    if (pages_per_seq <= 0 || pages_per_seq > 0x7fffffffll || words < (max_nodes + 63) / 64 || words > kPlanMaxWords) return AWEQ_ERR_SHAPE;
    if (n_seq == 0 || max_tokens == 0) return AWEQ_OK;
    if (!q || !out || !own_len || !start || !mask || !page_table || (prefix_len && !prefix_pages)) return AWEQ_ERR_NULL;
    const long long row = (long long)n_heads * cache->head_dim;
    if (!aligned(q, 16) || !aligned(out, 16) || ldq < row || ldo < row || ldq % 8 || ldo % 8 || ld_table < pages_per_seq ||
        !aligned(prefix_pages, 4) || !aligned(page_table, 4) || !aligned(own_len, 4) || !aligned(start, 4) || !aligned(pos, 4) || !aligned(mask, 8))
        return AWEQ_ERR_ALIGN;
    rc = check_ws(ws, ws_bytes, tree_attention_ws_bytes(cache, prefix_len, max_own, n_seq, max_tokens, max_nodes, n_heads));
    if (rc != AWEQ_OK) return rc;
    AWEQ_LOGF("aweq_tree_attention seqs=%lld tokens=%lld heads=%d kv_heads=%d head_dim=%d prefix=%lld max_own=%lld\n", n_seq, max_tokens, n_heads,
              cache->n_kv_heads, cache->head_dim, prefix_len, max_own);
    TreeArgs a = {};
    a.q = reinterpret_cast<const uint16_t *>(q); a.ck = reinterpret_cast<const uint16_t *>(cache->k);
    a.cv = reinterpret_cast<const uint16_t *>(cache->v); a.out = reinterpret_cast<uint16_t *>(out);
    a.ldq = ldq; a.ldo = ldo; a.n_pages = cache->n_pages; a.page_stride = cache->page_stride;
    a.token_stride = cache->token_stride; a.head_stride = cache->head_stride; a.page_size = cache->page_size;
    a.n_kv = cache->n_kv_heads; a.head_dim = cache->head_dim; a.n_heads = n_heads; a.words = words; a.max_nodes = max_nodes;
    a.max_tokens = (int)max_tokens; a.n_seq = (int)n_seq; a.prefix_pages = prefix_pages; a.page_table = page_table;
    a.own_len = own_len; a.start = start; a.pos = pos; a.first = first; a.mask = mask; a.prefix_len = prefix_len; a.pages_per_seq = pages_per_seq;
    a.ld_table = ld_table; a.max_own = max_own; a.scale = scale; a.st = st;
    return run_tree_attention(a, cache, ws, (cudaStream_t)stream);
}

aweq_status aweq_tree_attention(const void *q, long long ldq, const aweq_kv_cache *cache, const int *prefix_pages, long long prefix_len,
                                const int *page_table, long long pages_per_seq, long long ld_table, const int *own_len, const int *start,
                                const long long *mask, int words, long long max_own, long long n_seq, long long max_tokens, int max_nodes,
                                int n_heads, float scale, void *out, long long ldo, void *ws, size_t ws_bytes, aweq_dev_status *st,
                                void *stream)
{
    return tree_attention(q, ldq, cache, prefix_pages, prefix_len, page_table, pages_per_seq, ld_table, own_len, start, nullptr, 0, mask, words,
                          max_own, n_seq, max_tokens, max_nodes, n_heads, scale, out, ldo, ws, ws_bytes, st, stream);
}

aweq_status aweq_tree_attention_planned(const void *q, long long ldq, const aweq_kv_cache *cache, const int *prefix_pages, long long prefix_len,
                                        const int *page_table, long long pages_per_seq, long long ld_table, const int *own_len,
                                        const int *start, const int *pos, long long first, const long long *mask, int words, long long max_own,
                                        long long n_seq, long long max_tokens, int max_nodes, int n_heads, float scale, void *out,
                                        long long ldo, void *ws, size_t ws_bytes, aweq_dev_status *st, void *stream)
{
    if (first < 0 || first > 0x7fffffffll) return AWEQ_ERR_SHAPE;
    if (!pos && max_tokens > 0) return AWEQ_ERR_NULL;
    return tree_attention(q, ldq, cache, prefix_pages, prefix_len, page_table, pages_per_seq, ld_table, own_len, start, pos, first, mask, words,
                          max_own, n_seq, max_tokens, max_nodes, n_heads, scale, out, ldo, ws, ws_bytes, st, stream);
}

}  // extern "C"
