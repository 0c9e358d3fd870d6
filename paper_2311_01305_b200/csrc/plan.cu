// What a step of serving needs to know and to put right about the paged cache: aweq_kv_plan (pages, slots, positions and
// tree masks from request lengths) and aweq_kv_accept (an accepted path's keys and values to their places).
#include "common.cuh"
#include "kernels.h"

namespace aweq {

// What the tokens of a sequence and its page moves need.
struct PlanSeq {
    int start, held, have, want;               // first token, keys before, pages before and after
    int granted, take, give, after;            // new pages it gets, their and the returned pages' offsets in the ring, keys after
};
constexpr int kPlanThreads = 256, kPlanShared = 1024;      // sequences whose PlanSeq fit a CTA's shared memory

__device__ __forceinline__ int plan_pages(int keys, int page_size) { return (int)(((unsigned)keys + (unsigned)page_size - 1) / (unsigned)page_size); }

// sums over the threads before this one, and over all
struct PlanSums { long long before, all; };
__device__ __forceinline__ PlanSums plan_scan(long long v, long long *sh)
{
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    long long x = v;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const long long y = __shfl_up_sync(0xffffffffu, x, o);
        if (lane >= o) x += y;
    }
    __syncthreads();                           // (sh may still be read by the scan before)
    if (lane == 31) sh[warp] = x;
    __syncthreads();
    PlanSums r = {x - v, 0};
#pragma unroll
    for (int i = 0; i < kPlanThreads / 32; ++i) {
        if (i < warp) r.before += sh[i];
        r.all += sh[i];
    }
    return r;
}

// The ring's counters; such as cannot be (`bad`): an empty ring.
struct PlanRing { long long taken, given; bool bad; };
__device__ __forceinline__ PlanRing plan_state(const KvPlanArgs &a)
{
    const long long taken = a.state[0], given = a.state[1];
    const bool bad = taken < 0 || given < taken || given - taken > a.n_pages;
    return {bad ? 0 : taken, bad ? 0 : given, bad};
}

// The sequences' tokens and pages; every thread gets the totals.  `lead`: the one CTA that counts and writes what the caller sees.
struct PlanTotals { int tokens; long long taken, given; };      // tokens; the ring's counters after the step
__device__ __forceinline__ PlanTotals plan_sequences(const KvPlanArgs &a, long long taken, long long given, PlanSeq *into, long long *sh, bool lead)
{
    const long long cap = min(a.pages_per_seq * a.page_size, 0x7fffffffll);
    const long long free = given - taken;
    long long tokens = 0, more_before = 0, less_before = 0;
    for (int b0 = 0; b0 < (int)a.n_seq; b0 += kPlanThreads) {
        const int b = b0 + (int)threadIdx.x;
        const bool in = b < (int)a.n_seq;
        const int asked_held = in ? a.held[b] : 0, asked = in ? a.change[b] : 0;
        const int held = (int)(asked_held < 0 ? 0 : min((long long)asked_held, cap));
        int fresh = asked > 0 ? (int)min((long long)asked, cap - held) : 0;
        const int drop = asked < 0 ? (int)min(-(long long)asked, (long long)held) : 0;
        bool bad = held != asked_held || (asked > 0 ? fresh != asked : (long long)drop != -(long long)asked);
        // the tokens' places end where the rows do
        const PlanSums t = plan_scan(fresh, sh);
        const long long start = min(tokens + t.before, a.max_tokens);
        const int kept = (int)min((long long)fresh, a.max_tokens - start);
        bad |= kept != fresh;
        fresh = kept;
        const int have = plan_pages(held, a.page_size);
        int after = held + fresh - drop, want = plan_pages(after, a.page_size);
        const int more = max(want - have, 0), less = max(have - want, 0);
        // (no sequence asks for or has more than the pool: both sums in one, 32 bits each)
        const PlanSums m = plan_scan((long long)min((long long)more, a.n_pages) << 32 | min((long long)less, a.n_pages), sh);
        const long long take = more_before + (m.before >> 32), give = less_before + (m.before & 0xffffffffll);
        const int granted = (int)min((long long)more, max(free - take, 0ll));
        if (granted < more) {
            bad = true;
            want = have + granted;
            after = (int)min((long long)after, (long long)want * a.page_size);
        }
        // pages given back beyond what the ring holds are lost, and counted
        bad |= less > 0 && give + less > a.n_pages - free;
        if (in) {
            into[b] = {(int)start, held, have, want, granted, (int)min(take, a.n_pages), (int)min(give, a.n_pages), after};
            if (lead) {
                a.own_len[b] = after;
                a.start[b] = (int)start;
                if (bad && a.st) atomicAdd(&a.st->out_of_range, 1ull);
            }
        }
        tokens = min(tokens + t.all, a.max_tokens);
        more_before += m.all >> 32;
        less_before += m.all & 0xffffffffll;
    }
    if (lead && threadIdx.x == 0) a.start[a.n_seq] = (int)tokens;
    return {(int)tokens, taken + min(more_before, free), given + min(less_before, a.n_pages - free)};
}

// A page of the ring for a sequence's p'th page, -1 where there is none.
__device__ __forceinline__ int plan_ring(const KvPlanArgs &a, long long taken, const PlanSeq &s, int p)
{
    const int i = p - s.have;
    if (i >= s.granted) return -1;
    const int page = a.ring[(taken + s.take + i) % a.n_pages];
    return page < 0 || page >= a.n_pages ? -1 : page;
}

// Page moves (a warp per sequence) and tokens (four a thread), shared out over the grid.
__device__ __forceinline__ void plan_fill(const KvPlanArgs &a, long long taken, long long given, const PlanSeq *seqs, int total)
{
    const int n_seq = (int)a.n_seq, lane = threadIdx.x & 31;
    const long long free = given - taken;
    for (int b = blockIdx.x * (kPlanThreads / 32) + (threadIdx.x >> 5); b < n_seq; b += gridDim.x * (kPlanThreads / 32)) {
        const PlanSeq s = seqs[b];
        int *const row = a.page_table + (long long)b * a.ld_table;
        for (int p = s.have + lane; p < s.want; p += 32) {
            const int page = plan_ring(a, taken, s, p);
            row[p] = page;
            if (page < 0 && a.st) atomicAdd(&a.st->out_of_range, 1ull);
        }
        for (int p = s.want + lane; p < s.have; p += 32) {
            const long long at = s.give + (p - s.want);
            if (at < a.n_pages - free) a.ring[(given + at) % a.n_pages] = row[p];
            row[p] = -1;
        }
    }
    const int quads = (int)((a.max_tokens + 3) / 4);
    for (int i = blockIdx.x * kPlanThreads + threadIdx.x; i < quads; i += gridDim.x * kPlanThreads) {
        const int t0 = i * 4;
        int seq[4], pos[4];
        long long slot[4];
        // the last sequence that starts at or before t0 (of several with the same start, the last: the others are empty)
        int b = 0;
        if (t0 < total) {
            int n = n_seq;
            while (n > 1) {
                const int half = n >> 1;
                if (seqs[b + half].start <= t0) b += half;
                n -= half;
            }
        }
        PlanSeq s = seqs[b];
        int end = b + 1 < n_seq ? seqs[b + 1].start : total;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int t = t0 + j;
            seq[j] = pos[j] = -1;
            slot[j] = -1;
            if (t >= total) {
                if (a.mask && t < a.max_tokens)
                    for (int w = 0; w < a.words; ++w) a.mask[(long long)t * a.words + w] = 0;
                continue;
            }
            while (t >= end) {
                s = seqs[++b];
                end = b + 1 < n_seq ? seqs[b + 1].start : total;
            }
            const int node = t - s.start, key = s.held + node;
            int depth = node;
            if (a.mask) {
                // the node and those above it; a parent is a node before its child
                unsigned long long bits[kPlanMaxWords] = {};
                int at = node;
                depth = 0;
                if (node >> 6 >= a.words) {
                    if (a.st) atomicAdd(&a.st->out_of_range, 1ull);
                } else for (;;) {
#pragma unroll
                    for (int w = 0; w < kPlanMaxWords; ++w)
                        if (at >> 6 == w) bits[w] |= 1ull << (at & 63);
                    const int up = a.parent[s.start + at];
                    const bool bad = up < -1 || up >= at;
                    if (bad && at == node && a.st) atomicAdd(&a.st->out_of_range, 1ull);
                    if (bad || up < 0) break;
                    at = up;
                    ++depth;
                }
#pragma unroll
                for (int w = 0; w < kPlanMaxWords; ++w)
                    if (w < a.words) a.mask[(long long)t * a.words + w] = (long long)bits[w];
            }
            seq[j] = b;
            pos[j] = (int)(a.first + s.held + depth);
            if (key < s.after) {
                const int p = (int)((unsigned)key / (unsigned)a.page_size), r = key - p * a.page_size;
                const int page = p < s.have ? a.page_table[(long long)b * a.ld_table + p] : plan_ring(a, taken, s, p);
                if (page >= 0 && page < a.n_pages) slot[j] = (long long)page * a.page_size + r;
            }
        }
        if (t0 + 4 <= a.max_tokens) {
            *reinterpret_cast<int4 *>(a.seq + t0) = make_int4(seq[0], seq[1], seq[2], seq[3]);
            *reinterpret_cast<int4 *>(a.pos + t0) = make_int4(pos[0], pos[1], pos[2], pos[3]);
            *reinterpret_cast<longlong2 *>(a.slot + t0) = make_longlong2(slot[0], slot[1]);
            *reinterpret_cast<longlong2 *>(a.slot + t0 + 2) = make_longlong2(slot[2], slot[3]);
        } else
            for (int j = 0; j < 4 && t0 + j < a.max_tokens; ++j) {
                a.seq[t0 + j] = seq[j];
                a.pos[t0 + j] = pos[j];
                a.slot[t0 + j] = slot[j];
            }
    }
}

// Up to kPlanShared sequences: every CTA works out the sequences for itself and fills its share, in one launch.  The ring's counters
// are set by the CTA that ends last, when all have read them.
__global__ void __launch_bounds__(kPlanThreads) kv_plan_kernel(const KvPlanArgs a, unsigned *ticket)
{
    __shared__ PlanSeq seqs[kPlanShared];
    __shared__ long long sh[kPlanThreads / 32];
    pdl_begin();
    const PlanRing ring = plan_state(a);
    const PlanTotals all = plan_sequences(a, ring.taken, ring.given, seqs, sh, blockIdx.x == 0);
    __syncthreads();
    plan_fill(a, ring.taken, ring.given, seqs, all.tokens);
    if (threadIdx.x == 0) {
        // (this CTA's threads read the counters before the barriers above)
        __threadfence();
        if (gridDim.x == 1 || atomicAdd(ticket, 1u) == gridDim.x - 1) {
            a.state[0] = all.taken;
            a.state[1] = all.given;
            if (ring.bad && a.st) atomicAdd(&a.st->out_of_range, 1ull);
            *ticket = 0;
        }
    }
}

// More sequences: one CTA works them out, a second launch fills.
struct PlanHead { long long taken, given; int tokens; };
__global__ void __launch_bounds__(kPlanThreads) kv_plan_sequences_kernel(const KvPlanArgs a, PlanHead *head, PlanSeq *seqs)
{
    __shared__ long long sh[kPlanThreads / 32];
    pdl_begin();
    const PlanRing ring = plan_state(a);
    const PlanTotals all = plan_sequences(a, ring.taken, ring.given, seqs, sh, true);
    __syncthreads();
    if (threadIdx.x == 0) {
        *head = {ring.taken, ring.given, all.tokens};
        a.state[0] = all.taken;
        a.state[1] = all.given;
        if (ring.bad && a.st) atomicAdd(&a.st->out_of_range, 1ull);
    }
}
__global__ void __launch_bounds__(kPlanThreads) kv_plan_fill_kernel(const KvPlanArgs a, const PlanHead *head, const PlanSeq *seqs)
{
    pdl_begin();
    plan_fill(a, head->taken, head->given, seqs, head->tokens);
}

size_t kv_plan_ws_bytes(long long n_seq) { return n_seq <= kPlanShared ? 256 : 256 + (size_t)n_seq * sizeof(PlanSeq); }

aweq_status run_kv_plan(const KvPlanArgs &a, void *ws, cudaStream_t stream)
{
    long long ctas = (a.max_tokens + 4 * kPlanThreads - 1) / (4 * kPlanThreads);
    const long long by_seq = (a.n_seq + 31) / 32;                              // (page moves: four sequences to a warp at least)
    if (ctas < by_seq) ctas = by_seq;
    if (ctas > kSmCount * 4) ctas = kSmCount * 4;
    unsigned char *const w = reinterpret_cast<unsigned char *>(ws);
    if (a.n_seq <= kPlanShared) {
        AWEQ_LAUNCH(kv_plan_kernel, dim3((unsigned)ctas), dim3(kPlanThreads), 0, stream, a, reinterpret_cast<unsigned *>(w));
        return AWEQ_OK;
    }
    PlanHead *const head = reinterpret_cast<PlanHead *>(w);
    PlanSeq *const seqs = reinterpret_cast<PlanSeq *>(w + 256);
    AWEQ_LAUNCH(kv_plan_sequences_kernel, dim3(1), dim3(kPlanThreads), 0, stream, a, head, seqs);
    AWEQ_LAUNCH(kv_plan_fill_kernel, dim3((unsigned)ctas), dim3(kPlanThreads), 0, stream, a, (const PlanHead *)head, (const PlanSeq *)seqs);
    return AWEQ_OK;
}

// ------------------------------------------------------------------ accept
// A thread moves one 16-byte piece of every row of a sequence's path, in the path's order.  Paths ascend, so a place is read before
// it is written (key path[j] = i is read for place j < i), whatever the piece: no thread needs another.
__global__ void __launch_bounds__(128) kv_accept_kernel(const KvAcceptArgs a, int pieces, int blocks)
{
    pdl_begin();
    const int b = blockIdx.x / blocks, i = (blockIdx.x - b * blocks) * 128 + threadIdx.x;
    const bool lead = i == 0;
    if (i >= 2 * pieces) return;
    const long long base = a.base[b], cap = a.pages_per_seq * a.page_size;
    const int asked = a.n_path[b];
    int n = min(max(asked, 0), a.max_path);
    bool bad = n != asked;
    if (base < 0 || base > cap) {
        n = 0;
        bad = true;
    }
    const int piece = i % pieces, per_head = a.head_dim / 8;
    uint16_t *const pool = (i < pieces ? a.ck : a.cv) + piece / per_head * a.head_stride + piece % per_head * 8;
    const int *const path = a.path + (long long)b * a.ld_path, *const row = a.page_table + (long long)b * a.ld_table;
    // element of the pool of a key, -1: nowhere
    auto place = [&](long long key) -> long long {
        if (key >= cap) return -1;
        const unsigned p = (unsigned)((unsigned long long)key / (unsigned)a.page_size);
        const int page = row[p];
        return page < 0 || page >= a.n_pages ? -1 : page * a.page_stride + (key - (long long)p * a.page_size) * a.token_stride;
    };
    constexpr int U = 8;
    int last = -1;
    bool on = true;
    for (int i0 = 0; i0 < n && on; i0 += U) {
        uint4 x[U];
        long long to[U];
        int node[U];
#pragma unroll
        for (int j = 0; j < U; ++j) node[j] = i0 + j < n ? path[i0 + j] : -1;
#pragma unroll
        for (int j = 0; j < U; ++j) {
            to[j] = -1;
            if (i0 + j >= n) continue;
            if (node[j] <= last) on = false;                    // (what follows a node that is out of order stays where it is)
            last = node[j];
            const long long from = on ? place(base + node[j]) : -1;
            if (on) to[j] = place(base + i0 + j);
            if (from < 0 || to[j] < 0) {
                on = false;
                to[j] = -1;
            }
            if (node[j] == i0 + j) to[j] = -1;
            if (to[j] >= 0) x[j] = *reinterpret_cast<const uint4 *>(pool + from);
        }
#pragma unroll
        for (int j = 0; j < U; ++j)
            if (to[j] >= 0) *reinterpret_cast<uint4 *>(pool + to[j]) = x[j];
    }
    if (lead && (bad || !on) && a.st) atomicAdd(&a.st->out_of_range, 1ull);
}

aweq_status run_kv_accept(const KvAcceptArgs &a, cudaStream_t stream)
{
    const int pieces = a.n_kv * (a.head_dim / 8);
    const int blocks = (2 * pieces + 127) / 128;
    AWEQ_LAUNCH(kv_accept_kernel, dim3((unsigned)(a.n_seq * blocks)), dim3(128), 0, stream, a, pieces, blocks);
    return AWEQ_OK;
}

}  // namespace aweq
