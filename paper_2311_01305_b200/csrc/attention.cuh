// Shared pieces of the attention over a prefix and a sequence's own keys (attention.cu has the overview): how the
// work is cut, the walk over a CTA's units, the arguments of the two kernels that compute.
#pragma once
#include <math_constants.h>

#include "common.cuh"
#include "kernels.h"

namespace aweq {

// How the work is cut (host; also sizes the scratch).
struct AttentionPlan {
    int tensor;                  // 1: the prefix by attention_tc.cu, 0: by attention.cu (the own keys always)
    int unit, pre_unit;          // keys of a unit of own keys / of the prefix
    int box;                     // tensor: keys of one copy (a unit is several, each inside a page)
    int dp;                      // head_dim padded to 64, 96 or 128
    int pre_tile, own_tile;      // rows of a prefix / own item
    int pre_rt, own_rt;          // row tiles per key head / per sequence and key head
    int pre_rec, own_rec;        // rows of a record
    int ctas;                    // grid of attention.cu's kernel
    int tc_ctas;                 // tensor: grid of attention_tc.cu's
    long long pre_tiles, pre_units, rows;
    // scratch: start of each sequence's own units, their number, the CTAs of the prefix (long long[n_seq + 2]); records
    size_t off_pre_o, off_pre_ml, off_own_o, off_own_ml, total;
};

__device__ __forceinline__ float exp2_fast(float x)
{
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}
// What a row's probabilities 2^(score - base) are relative to; m is its maximum so far, or lies a little below it.
//
// They are rounded to the 16-bit type for the product with v (their sum takes them unrounded), which leaves each within
// u = 2^-11 (fp16) or 2^-8 (bf16) of itself, as the output's own rounding does, as long as it is a normal number.  fp16 has
// those down to 2^-14 and nothing below 2^-25, and a million keys beside one large one may all lie there.  So fp16 ones
// are held 2^7 times as large; below 2^-21 of 2^m they are off by at most 2^-32 of it each.  (In binary32 m - 7 is m - 8 at
// the lowest, wherever m lies.)
constexpr float kProbabilityShift = 7.0f;
template <class D>
__device__ __forceinline__ float probability_base(float m) { return D::kBf16 ? m : m - kProbabilityShift; }
// An own length, clamped.  `count`: the one caller that reports it.  (Lengths may come from a launch of this library that is still
// running when a kernel starts: its first look at them is a plain load, which stays behind the wait; an invariant one need not.  A later
// look, at a place that hangs on lengths already read, may be one.)
__device__ __forceinline__ int clamp_length(const AttentionArgs &a, int len, bool count)
{
    const int most = (int)min(a.max_own, a.pages_per_seq * a.page_size);
    if (count && a.st && (len < 0 || len > most)) atomicAdd(&a.st->out_of_range, 1ull);
    return len < 0 ? 0 : min(len, most);
}
__device__ __forceinline__ int own_length(const AttentionArgs &a, long long b) { return clamp_length(a, __ldg(a.own_len + b), false); }
__device__ __forceinline__ int tiles_of(int len, int unit) { return (int)(((unsigned)len + (unsigned)unit - 1) / (unsigned)unit); }

// The units are dealt out in order, total / ctas to a CTA and one more to the first total % ctas.  (Divisions of 64 bits
// take hundreds of cycles: only where the numbers need them.)
__device__ __forceinline__ long long div_units(long long a, int b)
{
    return a >> 32 ? a / b : (long long)((uint32_t)a / (uint32_t)b);
}
struct AttentionDeal {
    long long each, more;        // units of a CTA, CTAs with one more
    int ctas;                    // those that have any
    __device__ __forceinline__ AttentionDeal(long long total, int most)
    {
        ctas = total < most ? (int)total : most;
        each = ctas ? div_units(total, ctas) : 0;
        more = total - each * ctas;
    }
    __device__ __forceinline__ long long first(int cta) const { return each * cta + (cta < more ? cta : more); }
    __device__ __forceinline__ int cta_of(long long u) const
    {
        const long long big = more * (each + 1);
        if ((each + 1) >> 31) return u < big ? (int)(u / (each + 1)) : (int)(more + (u - big) / each);
        return u < big ? (int)div_units(u, (int)(each + 1)) : (int)more + (int)div_units(u - big, (int)each);
    }
};

// What a unit is: the tile'th tile of the `len` keys of an item (row tile rt of key head kh, own: of sequence b).
struct alignas(16) AttentionUnit {
    int kh, rt, b, tile, len;
    int leave;                   // the CTA's last unit of this item
    int stop;                    // 1: the CTA's last unit, 2: nothing to compute
};

// The walk over a CTA's units by a warp: every lane knows the unit and looks up the page of a key.
template <bool OWN>
struct AttentionWalk {
    AttentionUnit at;
    int tiles, next_len;         // of the item; length of the sequence after this one (its load is long under way when needed)
    __device__ __forceinline__ void advance(const AttentionArgs &a, const AttentionPlan &p)
    {
        if (++at.tile < tiles) return;
        at.tile = 0;
        if (++at.rt < (OWN ? p.own_rt : p.pre_rt)) return;
        at.rt = 0;
        if (++at.kh < a.n_kv || !OWN) return;
        at.kh = 0;
        const int n_seq = (int)a.n_seq;
        do {                                                    // sequences without keys have no units
            ++at.b;
            at.len = next_len;
            tiles = tiles_of(at.len, p.unit);
            next_len = at.b + 1 < n_seq ? own_length(a, at.b + 1) : 0;
        } while (tiles == 0 && at.b + 1 < n_seq);
    }
    __device__ __forceinline__ bool has(const AttentionPlan &p, int r) const { return at.tile * (OWN ? p.unit : p.pre_unit) + r < at.len; }
    // entry of the page list for the unit's r'th key, if there is such a key; not looked at here, so that the load can fly
    // (a prefix' page list lies where the launch knows it: a plain load)
    __device__ __forceinline__ int entry(const AttentionArgs &a, const AttentionPlan &p, int r) const
    {
        const int *pages = (OWN ? a.page_table + (long long)at.b * a.ld_table : a.prefix_pages) + (unsigned)(at.tile * (OWN ? p.unit : p.pre_unit) + r) / (unsigned)a.page_size;
        return has(p, r) ? OWN ? __ldg(pages) : *pages : 0;
    }
};

__device__ __forceinline__ int given_length(const AttentionArgs &a, int b) { return b < (int)a.n_seq ? a.own_len[b] : 0; }
// Tiles of 32 sequences: the lane's own length and tiles, and the tiles before it.
__device__ __forceinline__ long long scan_tiles(const AttentionArgs &a, const AttentionPlan &p, int given, bool count, int *len, int *n)
{
    *len = clamp_length(a, given, count);
    *n = tiles_of(*len, p.unit);
    int sum = *n;                                               // 32 lengths of at most 2^31 keys: below 2^31 tiles
#pragma unroll
    for (int x = 1; x < 32; x <<= 1) {
        const int y = __shfl_up_sync(0xffffffffu, sum, x);
        if ((int)(threadIdx.x & 31) >= x) sum += y;
    }
    return (long long)(sum - *n);
}
// The number of own units; every warp computes it.  `lead`: the one warp of the grid that counts bad lengths and leaves the
// starts of the sequences for the join.
__device__ __forceinline__ long long own_units(const AttentionArgs &a, const AttentionPlan &p, bool lead, long long *start)
{
    const int lane = threadIdx.x & 31, n_seq = (int)a.n_seq, per_seq = a.n_kv * p.own_rt;
    long long total = 0;
    int given = given_length(a, lane);
    for (int b0 = 0; b0 < n_seq; b0 += 32) {
        const int now = given;
        given = given_length(a, b0 + 32 + lane);                // (under way while this one is taken)
        int len, n;
        const long long before = scan_tiles(a, p, now, lead, &len, &n);
        if (lead && b0 + lane < n_seq) start[b0 + lane] = (total + before) * per_seq;
        total += __shfl_sync(0xffffffffu, before + n, 31);
    }
    return total * per_seq;
}

__device__ __forceinline__ bool bad_page(const AttentionArgs &a, int page) { return page < 0 || page >= a.n_pages; }
// A bad entry of a page list counts once: where its first key (row 0 of the page) is met by the first row tile of the first key
// head.  (The row is at hand: another division there cost 1 us at 32 x (2048 + 300) keys.)
__device__ __forceinline__ void count_bad_page(const AttentionArgs &a, int kh, int rt, unsigned row)
{
    if (((unsigned)(kh | rt) | row) == 0 && a.st) atomicAdd(&a.st->out_of_range, 1ull);
}

// A warp finds the first unit of CTA `cta` of `ctas` (every lane gets the same) and the number of its units.
template <bool OWN>
__device__ __forceinline__ int attention_begin(const AttentionArgs &a, const AttentionPlan &p, int cta, int ctas, long long total,
                                               AttentionWalk<OWN> &w)
{
    w.at = {};
    const AttentionDeal deal(total, ctas);
    if (cta >= deal.ctas) return 0;
    const long long u0 = deal.first(cta);
    if (!OWN) {
        const int item = (int)div_units(u0, (int)p.pre_tiles);
        w.at.kh = item / p.pre_rt;
        w.at.rt = item % p.pre_rt;
        w.at.tile = (int)(u0 - item * p.pre_tiles);
        w.at.len = (int)a.prefix_len;
        w.tiles = (int)p.pre_tiles;
        return (int)(deal.first(cta + 1) - u0);
    }
    const int lane = threadIdx.x & 31, n_seq = (int)a.n_seq, per_seq = a.n_kv * p.own_rt;
    long long passed = 0;
    int given = given_length(a, lane);
    for (int b0 = 0;; b0 += 32) {
        const int now = given;
        given = given_length(a, b0 + 32 + lane);
        int len, n;
        const long long mine = passed + scan_tiles(a, p, now, false, &len, &n) * per_seq;
        const uint32_t here = __ballot_sync(0xffffffffu, u0 >= mine && u0 < mine + (long long)n * per_seq);
        if (here) {
            const int src = __ffs(here) - 1, within = (int)(u0 - __shfl_sync(0xffffffffu, mine, src));
            w.tiles = __shfl_sync(0xffffffffu, n, src);
            const int item = within / w.tiles;
            w.at.b = b0 + src;
            w.at.kh = item / p.own_rt;
            w.at.rt = item % p.own_rt;
            w.at.tile = within - item * w.tiles;
            w.at.len = __shfl_sync(0xffffffffu, len, src);
            w.next_len = src < 31 ? __shfl_sync(0xffffffffu, len, src + 1) : w.at.b + 1 < n_seq ? own_length(a, w.at.b + 1) : 0;
            break;
        }
        passed = __shfl_sync(0xffffffffu, mine + (long long)n * per_seq, 31);
    }
    return (int)(deal.first(cta + 1) - u0);
}

// attention_tc.cu
aweq_status run_attention_tc(const AttentionArgs &a, const AttentionPlan &p, aweq_dtype dt, unsigned char *ws, cudaStream_t stream);

}  // namespace aweq
