// Shared pieces of the attention of drafted trees (tree.cu has the overview): how the work is cut and walked.
#pragma once
#include <math_constants.h>

#include "attention.cuh"
#include "common.cuh"
#include "kernels.h"

namespace aweq {

struct TreePlan {
    int two;                     // 1: an item has two tiles of rows on the same keys; 0: one, whose units alternate between two sums
    int group, part, rows;       // heads to a key head; rows of a tile: whole tokens, up to 128; rows of an item: one tile or two
    int unit, box;               // keys of a unit, of one tiled copy (0: 16-byte copies)
    int ctas, pre_rt, pre_tiles; // grid; most row tiles of the prefix; units of a prefix item
    int pre_rec, own_rec;        // rows of a record, of one sum each
    // scratch: the totals, per sequence its first own unit and item (TreeFirst[n_seq]), every token's sequence; records
    size_t off_seq, off_pre_o, off_pre_ml, off_own_o, off_own_ml, total;
};
struct alignas(16) TreeFirst { long long unit; int item, tiles, t0; short nodes, placed; int base, n_rt; };
// How the units are dealt: evenly, an item counting `change` units more than it has, ahead of its own (the record that a CTA writes when
// it leaves an item takes as long as two or three units: 16 trees of 24 nodes after 512 + 2100 keys 56 us without, 50 with two; one and
// three are within 2 % of two over seven shapes, but for 128 short items, where one would be 4 % faster).
// pre, own: units of both kinds so counted; each, more: units of a CTA, CTAs with one more.
struct alignas(16) TreeTotals { long long pre, own, each, more; int tokens, pre_rt, ctas, change; };
constexpr int kTrChange = 2, kTrChangeFrom = 4;     // with as many units to a CTA or more

// A sequence's new tokens and the keys before them, clamped.
// base: key of node 0 (below zero: the first nodes have none); placed: the nodes before the first one behind the last key; ctx: keys before them
struct TreeSeq { int t0, t1, nodes, placed, ctx, base; bool bad; };
// Of 32 sequences, a lane each (b: the lane's).  A start below one before it counts as that one, so that no token belongs to two
// sequences and the rows of all are no more than the tokens', which the scratch is made for.  top: where the sequences before these end.
__device__ __forceinline__ TreeSeq tree_load(const TreeArgs &a, int b, int top)
{
    const bool in = b < a.n_seq;
    const int s0 = in ? a.start[b] : 0, s1 = in ? a.start[b + 1] : 0, len = in ? a.own_len[b] : 0;
    const int cap = (int)min(a.max_own, a.pages_per_seq * a.page_size);
    TreeSeq s;
    s.t0 = min(max(s0, 0), a.max_tokens);
    s.t1 = min(max(s1, 0), a.max_tokens);
    if (__any_sync(0xffffffffu, in && (s.t0 < top || s.t1 < s.t0))) {
        s.t0 = max(s.t0, top);
#pragma unroll 1
        for (int x = 1; x < 32; x <<= 1) s.t0 = max(s.t0, __shfl_up_sync(0xffffffffu, s.t0, x));      // (the lowest lanes get their own)
        s.t1 = max(s.t0, s.t1);
    }
    const int l = min(max(len, 0), cap);
    s.nodes = min(s.t1 - s.t0, a.max_nodes);
    // the last keys are those of all the sequence's tokens, also where some are not computed or some keys are beyond what there may be;
    // or the tokens' positions say where theirs begin (a length short of them then leaves the last without a key)
    const int tokens = s.t1 - s.t0;
    const long long base = a.pos ? (in && tokens ? a.pos[s.t0] - a.first : l) : (long long)max(len, 0) - tokens;
    s.base = (int)min(max(base, -64ll * kPlanMaxWords), (long long)l);
    s.placed = min(s.nodes, l - s.base);
    s.ctx = max(s.base, 0);
    s.bad = s.t0 != s0 || s.t1 != s1 || s.nodes != s.t1 - s.t0 || l != len || base < 0 || (tokens && base + tokens > l);
    return in ? s : TreeSeq{0, 0, 0, 0, 0, 0, false};
}
// Where the 32 sequences from b0 on end.
__device__ __forceinline__ int tree_end(const TreeArgs &a, const TreeSeq &s, int b0, int top)
{
    return max(top, __shfl_sync(0xffffffffu, s.t1, min(31, max(a.n_seq - 1 - b0, 0))));
}
__device__ __forceinline__ int tree_tokens(const TreeArgs &a) { return min(max(a.start[a.n_seq], 0), a.max_tokens); }
__device__ __forceinline__ int tree_tiles(int n, int of) { return (int)(((unsigned)n + (unsigned)of - 1) / (unsigned)of); }

// own units and items of 32 sequences, and the items that have units: the lane's, and those before it
struct TreeScan {
    long long units, unit0;
    int items, item0, busy, busy0;
    __device__ __forceinline__ TreeScan counted(int change) const           // units as they are dealt
    {
        TreeScan r = *this;
        r.units += (long long)change * busy;
        r.unit0 += (long long)change * busy0;
        return r;
    }
};
__device__ __forceinline__ TreeScan tree_scan(const TreeArgs &a, const TreePlan &p, const TreeSeq &s)
{
    const int lane = threadIdx.x & 31;
    TreeScan r;
    r.items = a.n_kv * tree_tiles(s.nodes * p.group, p.rows);
    r.units = (long long)r.items * tree_tiles(s.ctx, p.unit);
    r.busy = s.ctx > 0 ? r.items : 0;
    long long u = r.units;
    int i = r.items, k = r.busy;
#pragma unroll 1
    for (int x = 1; x < 32; x <<= 1) {
        const long long v = __shfl_up_sync(0xffffffffu, u, x);
        const int w = __shfl_up_sync(0xffffffffu, i, x), y = __shfl_up_sync(0xffffffffu, k, x);
        if (lane >= x) { u += v; i += w; k += y; }
    }
    r.busy0 = k - r.busy;
    r.unit0 = u - r.units;
    r.item0 = i - r.items;
    return r;
}
// All units; every CTA computes them for itself.  s0, c0: what the lane has of the first 32 sequences.
__device__ __forceinline__ TreeTotals tree_totals(const TreeArgs &a, const TreePlan &p, TreeSeq &s0, TreeScan &c0)
{
    TreeTotals t;
    t.tokens = tree_tokens(a);
    t.own = 0;
    long long busy = 0;
    int top = 0;
    for (int b0 = 0; b0 < a.n_seq; b0 += 32) {
        const TreeSeq s = tree_load(a, b0 + (int)(threadIdx.x & 31), top);
        top = tree_end(a, s, b0, top);
        const TreeScan c = tree_scan(a, p, s);
        if (b0 == 0) {
            s0 = s;
            c0 = c;
        }
        t.own += __shfl_sync(0xffffffffu, c.unit0 + c.units, 31);
        busy += __shfl_sync(0xffffffffu, c.busy0 + c.busy, 31);
    }
    t.pre_rt = tree_tiles(t.tokens * p.group, p.rows);
    const long long items = p.pre_tiles ? (long long)a.n_kv * t.pre_rt : 0;
    t.change = t.own + items * p.pre_tiles >= (long long)kTrChangeFrom * p.ctas ? kTrChange : 0;
    t.own += busy * t.change;
    t.pre = items * (p.pre_tiles + t.change);
    c0 = c0.counted(t.change);
    return t;
}
// What the join needs, in scratch: every ctas'th sequence's first unit and item, and the sequence of its tokens.  Lengths and starts out
// of range are counted here, once.
__device__ __forceinline__ void tree_leave(const TreeArgs &a, const TreePlan &p, unsigned char *ws, int cta, int change)
{
    const int lane = threadIdx.x & 31;
    TreeFirst *const first = reinterpret_cast<TreeFirst *>(ws + sizeof(TreeTotals));
    int *const seq_of = reinterpret_cast<int *>(ws + p.off_seq);
    long long units = 0;
    int items = 0, top = 0;
    for (int b0 = 0; b0 < a.n_seq; b0 += 32) {
        const TreeSeq s = tree_load(a, b0 + lane, top);
        top = tree_end(a, s, b0, top);
        const TreeScan c = tree_scan(a, p, s).counted(change);
        const bool mine = b0 + lane < a.n_seq && (unsigned)(b0 + lane) % (unsigned)p.ctas == (unsigned)cta;
        if (mine) {
            first[b0 + lane] = {units + c.unit0, items + c.item0, tree_tiles(s.ctx, p.unit), s.t0, (short)s.nodes, (short)s.placed, s.base,
                               tree_tiles(s.nodes * p.group, p.rows)};
            if (s.bad && a.st) atomicAdd(&a.st->out_of_range, 1ull);
        }
        for (uint32_t left = __ballot_sync(0xffffffffu, mine); left; left &= left - 1) {
            const int src = __ffs(left) - 1, b = b0 + src, t0 = __shfl_sync(0xffffffffu, s.t0, src), t1 = __shfl_sync(0xffffffffu, s.t1, src);
            for (int t = t0 + lane; t < t1; t += 32) seq_of[t] = b;
            if (b == 0)
                for (int t = lane; t < t0; t += 32) seq_of[t] = -1;         // (starts that do not begin at zero)
        }
        units += __shfl_sync(0xffffffffu, c.unit0 + c.units, 31);
        items += __shfl_sync(0xffffffffu, c.item0 + c.items, 31);
    }
}

// What a CTA has of an item: units tile .. tile + count - 1 of a segment's keys on one row tile of one key head.
struct alignas(16) TreeItem {
    int own, b, kh, rt;          // b: the sequence (own)
    int tile, count, len, rows;  // len: keys of the segment
    int t0, stop;                // first token of the rows; the CTA's last item
    long long rec;               // first row of its record
};

// The walk over a CTA's items by a warp (every lane knows the item): prefix items first, then each sequence's, row tiles inside
// key heads.
struct TreeWalk {
    int own, b, kh, rt, tile, tiles, n_rt, len, t0, n_tok, item;     // t0, n_tok: the tokens whose rows they are
    int ahead, top;                                                  // counted units before the first; where the sequences so far end
    __device__ __forceinline__ void take(const TreePlan &p, const TreeSeq &s, int src)
    {
        t0 = __shfl_sync(0xffffffffu, s.t0, src);
        top = __shfl_sync(0xffffffffu, s.t1, src);
        n_tok = __shfl_sync(0xffffffffu, s.nodes, src);
        len = __shfl_sync(0xffffffffu, s.ctx, src);
        tiles = tree_tiles(len, p.unit);
        n_rt = tree_tiles(n_tok * p.group, p.rows);
    }
    __device__ __forceinline__ void enter(const TreeArgs &a, const TreePlan &p, int to)        // the next sequence with units
    {
        own = 1;
        for (int b0 = to;; b0 += 32) {
            const TreeSeq s = tree_load(a, b0 + (int)(threadIdx.x & 31), top);
            const TreeScan c = tree_scan(a, p, s);
            const uint32_t here = __ballot_sync(0xffffffffu, c.units > 0);
            if (here || b0 + 32 >= a.n_seq) {
                const int src = here ? __ffs(here) - 1 : 0;
                b = b0 + src;
                item += __shfl_sync(0xffffffffu, c.item0, src);
                take(p, s, src);
                return;
            }
            item += __shfl_sync(0xffffffffu, c.item0 + c.items, 31);
            top = tree_end(a, s, b0, top);
        }
    }
    __device__ __forceinline__ void place(int counted, int change)
    {
        tile = max(counted - change, 0);
        ahead = max(change - counted, 0);
    }
    __device__ __forceinline__ void begin(const TreeArgs &a, const TreePlan &p, const TreeTotals &t, long long u0, const TreeSeq &s0, const TreeScan &c0)
    {
        own = b = kh = rt = tile = tiles = n_rt = len = t0 = n_tok = item = ahead = top = 0;
        const int lane = threadIdx.x & 31;
        if (u0 < t.pre) {
            tiles = p.pre_tiles;
            len = (int)a.prefix_len;
            n_tok = t.tokens;
            n_rt = tree_tiles(n_tok * p.group, p.rows);
            item = (int)div_units(u0, tiles + t.change);
            place((int)(u0 - (long long)item * (tiles + t.change)), t.change);
            kh = item / n_rt;
            rt = item - kh * n_rt;
            return;
        }
        const long long u = u0 - t.pre;
        long long passed = 0;
        int items = 0;
        for (int b0 = 0; b0 < a.n_seq; b0 += 32) {
            const TreeSeq s = b0 ? tree_load(a, b0 + lane, top) : s0;
            const TreeScan c = b0 ? tree_scan(a, p, s).counted(t.change) : c0;
            const uint32_t here = __ballot_sync(0xffffffffu, u >= passed + c.unit0 && u < passed + c.unit0 + c.units);
            if (here) {
                const int src = __ffs(here) - 1;
                own = 1;
                b = b0 + src;
                const long long within = u - passed - __shfl_sync(0xffffffffu, c.unit0, src);
                take(p, s, src);
                const int i = (int)div_units(within, tiles + t.change);
                place((int)(within - (long long)i * (tiles + t.change)), t.change);
                kh = i / n_rt;
                rt = i - kh * n_rt;
                item = items + __shfl_sync(0xffffffffu, c.item0, src) + i;
                return;
            }
            passed += __shfl_sync(0xffffffffu, c.unit0 + c.units, 31);
            items += __shfl_sync(0xffffffffu, c.item0 + c.items, 31);
            top = tree_end(a, s, b0, top);
        }
    }
    __device__ __forceinline__ void next_item(const TreeArgs &a, const TreePlan &p)
    {
        tile = 0;
        ++item;
        if (++rt < n_rt) return;
        rt = 0;
        if (++kh < a.n_kv) return;
        kh = 0;
        if (!own) item = 0;
        enter(a, p, own ? b + 1 : 0);
    }
    __device__ __forceinline__ int rows(const TreePlan &p) const { return min(p.rows, n_tok * p.group - rt * p.rows); }
};

}  // namespace aweq
