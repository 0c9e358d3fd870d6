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
constexpr int kPlanThreads = 512, kPlanShared = 1024;      // sequences whose PlanSeq fit a CTA's shared memory

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
    constexpr int M = 2;                       // sequences of a thread, so that two scans serve a thousand
    for (int b0 = 0; b0 < (int)a.n_seq; b0 += M * kPlanThreads) {
        const int b1 = b0 + M * (int)threadIdx.x;
        int held[M], fresh[M], drop[M];
        bool bad[M];
        long long sum = 0;
#pragma unroll
        for (int i = 0; i < M; ++i) {
            const bool in = b1 + i < (int)a.n_seq;
            const int asked_held = in ? a.held[b1 + i] : 0, asked = in ? a.change[b1 + i] : 0;
            held[i] = (int)(asked_held < 0 ? 0 : min((long long)asked_held, cap));
            fresh[i] = asked > 0 ? (int)min((long long)asked, cap - held[i]) : 0;
            drop[i] = asked < 0 ? (int)min(-(long long)asked, (long long)held[i]) : 0;
            bad[i] = held[i] != asked_held || (asked > 0 ? fresh[i] != asked : (long long)drop[i] != -(long long)asked);
            sum += fresh[i];
        }
        // the tokens' places end where the rows do
        const PlanSums t = plan_scan(sum, sh);
        long long at = tokens + t.before, pages = 0;
        int start[M], have[M], want[M], after[M];
#pragma unroll
        for (int i = 0; i < M; ++i) {
            const long long from = min(at, a.max_tokens);
            const int kept = (int)min((long long)fresh[i], a.max_tokens - from);
            at += fresh[i];
            start[i] = (int)from;
            bad[i] |= kept != fresh[i];
            have[i] = plan_pages(held[i], a.page_size);
            after[i] = held[i] + kept - drop[i];
            want[i] = plan_pages(after[i], a.page_size);
            // (both sums in one: pages taken are no more than the tokens, 31 bits; a thousand sequences' pages put back, of 2^22 each, 33)
            pages += (long long)((unsigned long long)min((long long)max(want[i] - have[i], 0), a.n_pages) << 33) + min((long long)max(have[i] - want[i], 0), a.n_pages);
        }
        const PlanSums m = plan_scan(pages, sh);
        auto taken_of = [](long long sums) { return (long long)((unsigned long long)sums >> 33); };
        auto given_of = [](long long sums) { return sums & 0x1ffffffffll; };
        long long take = more_before + taken_of(m.before), give = less_before + given_of(m.before);
#pragma unroll
        for (int i = 0; i < M; ++i) {
            const int more = max(want[i] - have[i], 0), less = max(have[i] - want[i], 0);
            const int granted = (int)min((long long)more, max(free - take, 0ll));
            if (granted < more) {
                bad[i] = true;
                want[i] = have[i] + granted;
                after[i] = (int)min((long long)after[i], (long long)want[i] * a.page_size);
            }
            // pages given back beyond what the ring holds are lost, and counted
            bad[i] |= less > 0 && give + less > a.n_pages - free;
            if (b1 + i < (int)a.n_seq) {
                into[b1 + i] = {start[i], held[i], have[i], want[i], granted, (int)min(take, a.n_pages), (int)min(give, a.n_pages), after[i]};
                if (lead) {
                    a.own_len[b1 + i] = after[i];
                    a.start[b1 + i] = start[i];
                    if (bad[i] && a.st) atomicAdd(&a.st->out_of_range, 1ull);
                }
            }
            take += min((long long)more, a.n_pages);
            give += min((long long)less, a.n_pages);
        }
        tokens = min(tokens + t.all, a.max_tokens);
        more_before += taken_of(m.all);
        less_before += given_of(m.all);
    }
    if (lead && threadIdx.x == 0) a.start[a.n_seq] = (int)tokens;
    return {(int)tokens, taken + min(more_before, free), given + min(less_before, a.n_pages - free)};
}

// Where the ring's next free page lies, and where the next one given back goes.
struct PlanEnds { int take, give, free; };
__device__ __forceinline__ PlanEnds plan_ends(const KvPlanArgs &a, long long taken, long long given)
{
    return {(int)(taken % a.n_pages), (int)(given % a.n_pages), (int)(given - taken)};
}
// (offsets are at most n_pages, ends below it)
__device__ __forceinline__ int plan_at(const KvPlanArgs &a, int end, int offset)
{
    const int i = end + offset, n = (int)a.n_pages;
    return i < n ? i : i - n;
}
// A page of the ring for a sequence's p'th page, -1 where there is none.
__device__ __forceinline__ int plan_ring(const KvPlanArgs &a, const PlanEnds &e, const PlanSeq &s, int p)
{
    const int i = p - s.have;
    if (i >= s.granted) return -1;
    const int page = a.ring[plan_at(a, e.take, s.take + i)];
    return page < 0 || page >= a.n_pages ? -1 : page;
}

// the last sequence that starts at or before token t (of several with the same start, the last: the others are empty)
__device__ __forceinline__ int plan_find(const PlanSeq *seqs, int n_seq, int t)
{
    int b = 0;
    for (int n = n_seq; n > 1;) {
        const int half = n >> 1;
        if (seqs[b + half].start <= t) b += half;
        n -= half;
    }
    return b;
}

// Page moves, a warp per sequence.
__device__ __forceinline__ void plan_pages_move(const KvPlanArgs &a, const PlanEnds &e, const PlanSeq *seqs)
{
    const int lane = threadIdx.x & 31;
    for (int b = blockIdx.x * (kPlanThreads / 32) + (threadIdx.x >> 5); b < (int)a.n_seq; b += gridDim.x * (kPlanThreads / 32)) {
        const PlanSeq s = seqs[b];
        int *const row = a.page_table + (long long)b * a.ld_table;
        for (int p = s.have + lane; p < s.want; p += 32) {
            const int page = plan_ring(a, e, s, p);
            row[p] = page;
            if (page < 0 && a.st) atomicAdd(&a.st->out_of_range, 1ull);
        }
        for (int p = s.want + lane; p < s.have; p += 32) {
            const long long at = (long long)s.give + (p - s.want);
            if (at < a.n_pages - e.free) a.ring[plan_at(a, e.give, (int)at)] = row[p];
            row[p] = -1;
        }
    }
}
// The page of a sequence's p'th, -1 where there is none.
__device__ __forceinline__ int plan_page(const KvPlanArgs &a, const PlanEnds &e, const PlanSeq &s, int b, int p)
{
    const int page = p < s.have ? a.page_table[(long long)b * a.ld_table + p] : plan_ring(a, e, s, p);
    return page >= 0 && page < a.n_pages ? page : -1;
}

// Tokens in a row, four to a thread (so that a warp's stores lie together: with eight the sectors came in halves, 22.5 us in the place
// of 16.5 for 1.6 million tokens): one search, one division, and a look-up for each page they touch; runs within a sequence, which nearly
// all are, without a test for every token (15 to 14 us; 60 % of the issue slots).
__device__ __forceinline__ void plan_tokens(const KvPlanArgs &a, const PlanEnds &e, const PlanSeq *seqs, int total)
{
    constexpr int M = 4;
    const bool wide = (reinterpret_cast<uintptr_t>(a.slot) & 31) == 0;
    const int n_seq = (int)a.n_seq, runs = (int)((a.max_tokens + M - 1) / M);
    for (int i = blockIdx.x * kPlanThreads + threadIdx.x; i < runs; i += gridDim.x * kPlanThreads) {
        const int t0 = i * M;
        int seq[M], pos[M];
        long long slot[M];
        int b = 0, key = 0, end = 0, p = 0, row = 0, page = -1;
        PlanSeq s = {};
        auto enter = [&](int t) {
            s = seqs[b];
            end = b + 1 < n_seq ? seqs[b + 1].start : total;
            key = s.held + t - s.start;
            p = (int)((unsigned)key / (unsigned)a.page_size);
            row = key - p * a.page_size;
            page = key < s.after ? plan_page(a, e, s, b, p) : -1;
        };
        if (t0 < total) {
            b = plan_find(seqs, n_seq, t0);
            enter(t0);
        }
        if (t0 + M <= end && key + M <= s.after && M <= a.page_size) {
            // of one sequence, all with a place, on one page or two
            const int next = row + M > a.page_size ? plan_page(a, e, s, b, p + 1) : -1;
            const long long at0 = (long long)page * a.page_size + row, at1 = ((long long)next - 1) * a.page_size + row;
#pragma unroll
            for (int j = 0; j < M; ++j) {
                seq[j] = b;
                pos[j] = (int)(a.first + key) + j;
                const bool here = row + j < a.page_size;
                slot[j] = (here ? page : next) < 0 ? -1 : (here ? at0 : at1) + j;
            }
        } else
#pragma unroll
        for (int j = 0; j < M; ++j) {
            const int t = t0 + j;
            seq[j] = pos[j] = -1;
            slot[j] = -1;
            if (t >= total) continue;
            if (t >= end) {
                do ++b;                        // (sequences without tokens lie between)
                while (b + 1 < n_seq && seqs[b + 1].start <= t);
                enter(t);
            }
            seq[j] = b;
            pos[j] = (int)(a.first + key);
            if (page >= 0 && key < s.after) slot[j] = (long long)page * a.page_size + row;
            ++key;
            if (++row == a.page_size) {
                row = 0;
                ++p;
                page = j + 1 < M && key < s.after && t + 1 < end ? plan_page(a, e, s, b, p) : -1;
            }
        }
        if (t0 + M <= a.max_tokens) {
            *reinterpret_cast<int4 *>(a.seq + t0) = make_int4(seq[0], seq[1], seq[2], seq[3]);
            *reinterpret_cast<int4 *>(a.pos + t0) = make_int4(pos[0], pos[1], pos[2], pos[3]);
            if (wide)
                asm volatile("st.global.v4.b64 [%0], {%1, %2, %3, %4};" ::"l"(a.slot + t0), "l"(slot[0]), "l"(slot[1]), "l"(slot[2]), "l"(slot[3]) : "memory");
            else {
                *reinterpret_cast<longlong2 *>(a.slot + t0) = make_longlong2(slot[0], slot[1]);
                *reinterpret_cast<longlong2 *>(a.slot + t0 + 2) = make_longlong2(slot[2], slot[3]);
            }
        } else
#pragma unroll
            for (int j = 0; j < M; ++j)
                if (t0 + j < a.max_tokens) {
                    a.seq[t0 + j] = seq[j];
                    a.pos[t0 + j] = pos[j];
                    a.slot[t0 + j] = slot[j];
                }
    }
}

// Nodes of trees, a thread each.  A node's way up is a chain of look-ups, so the parents of a CTA's nodes and of the nodes before them
// that a tree can reach lie in shared memory.
__device__ __forceinline__ void plan_nodes(const KvPlanArgs &a, const PlanEnds &e, const PlanSeq *seqs, int total, int *parents)
{
    constexpr int kBack = 64 * kPlanMaxWords;
    const int n_seq = (int)a.n_seq;
    for (long long t00 = (long long)blockIdx.x * kPlanThreads; t00 < a.max_tokens; t00 += (long long)gridDim.x * kPlanThreads) {
        const int t0 = (int)t00, t = t0 + (int)threadIdx.x;
        __syncthreads();
        for (int i = threadIdx.x; i < kBack + kPlanThreads; i += kPlanThreads) {
            const int from = t0 - kBack + i;
            parents[i] = from >= 0 && from < total ? a.parent[from] : -1;
        }
        __syncthreads();
        if (t >= a.max_tokens) continue;
        int seq = -1, pos = -1;
        long long slot = -1;
        unsigned long long bits[kPlanMaxWords] = {};
        if (t < total) {
            const int b = plan_find(seqs, n_seq, t);
            const PlanSeq s = seqs[b];
            const int node = t - s.start, *const mine = parents + kBack - node + (int)threadIdx.x;      // parents of the sequence's nodes
            int depth = 0;
            if (node >> 6 < a.words) {
                // the node and those above it; a parent is a node before its child
                for (int at = node;;) {
#pragma unroll
                    for (int w = 0; w < kPlanMaxWords; ++w)
                        if (at >> 6 == w) bits[w] |= 1ull << (at & 63);
                    const int up = mine[at];
                    const bool bad = up < -1 || up >= at;
                    if (bad && at == node && a.st) atomicAdd(&a.st->out_of_range, 1ull);
                    if (bad || up < 0) break;
                    at = up;
                    ++depth;
                }
            } else if (a.st) atomicAdd(&a.st->out_of_range, 1ull);
            seq = b;
            pos = (int)(a.first + s.held + depth);
            const int key = s.held + node, p = (int)((unsigned)key / (unsigned)a.page_size);
            const int page = key < s.after ? plan_page(a, e, s, b, p) : -1;
            if (page >= 0) slot = (long long)page * a.page_size + (key - p * a.page_size);
        }
        a.seq[t] = seq;
        a.pos[t] = pos;
        a.slot[t] = slot;
#pragma unroll
        for (int w = 0; w < kPlanMaxWords; ++w)
            if (w < a.words) a.mask[(long long)t * a.words + w] = (long long)bits[w];
    }
}

__device__ __forceinline__ void plan_fill(const KvPlanArgs &a, const PlanRing &ring, const PlanSeq *seqs, int total, int *parents)
{
    const PlanEnds e = plan_ends(a, ring.taken, ring.given);
    plan_pages_move(a, e, seqs);
    if (a.mask) plan_nodes(a, e, seqs, total, parents);
    else plan_tokens(a, e, seqs, total);
}

// Up to kPlanShared sequences: every CTA works out the sequences for itself and fills its share, in one launch.  Bound by latency:
// counters and lengths, two scans, then for each token search, page, stores; 64 trees 10 us by itself and 6.7 for
// giving back, 512 prompts (1.6 million tokens, 26 MB) 14 us, of which 4 are the stores' at a copy's rate and 5 the sequences'.  The ring's counters
// are set by the CTA that comes last, when all have read them.
__global__ void __launch_bounds__(kPlanThreads) kv_plan_kernel(const KvPlanArgs a, unsigned *ticket)
{
    __shared__ PlanSeq seqs[kPlanShared];
    __shared__ int parents[64 * kPlanMaxWords + kPlanThreads];
    __shared__ long long sh[kPlanThreads / 32];
    pdl_begin();
    const PlanRing ring = plan_state(a);
    const PlanTotals all = plan_sequences(a, ring.taken, ring.given, seqs, sh, blockIdx.x == 0);
    __syncthreads();
    // (this CTA's threads have read the counters; not at the end, where the fence would wait for the stores)
    if (threadIdx.x == 0) {
        __threadfence();
        if (gridDim.x == 1 || atomicAdd(ticket, 1u) == gridDim.x - 1) {
            a.state[0] = all.taken;
            a.state[1] = all.given;
            if (ring.bad && a.st) atomicAdd(&a.st->out_of_range, 1ull);
            *ticket = 0;
        }
    }
    plan_fill(a, ring, seqs, all.tokens, parents);
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
    __shared__ int parents[64 * kPlanMaxWords + kPlanThreads];
    pdl_begin();
    plan_fill(a, {head->taken, head->given, false}, seqs, head->tokens, parents);
}

// Scratch: the ticket, zero between calls; behind it, for more sequences than one launch serves, the head and the sequences.  (A word of its
// own, so that calls of both kinds may take turns.)
constexpr size_t kPlanHeadAt = 64, kPlanSeqsAt = 256;
size_t kv_plan_ws_bytes(long long n_seq) { return n_seq <= kPlanShared ? kPlanSeqsAt : kPlanSeqsAt + (size_t)n_seq * sizeof(PlanSeq); }

aweq_status run_kv_plan(const KvPlanArgs &a, void *ws, cudaStream_t stream)
{
    // every CTA works out the sequences for itself, so no more of them than the tokens (eight to a thread in two turns, nodes one) and the page moves
    // (a sequence to a warp) keep busy
    const int per = kPlanThreads * (a.mask ? 1 : 8);
    long long ctas = (a.max_tokens + per - 1) / per;
    const long long by_seq = (a.n_seq + kPlanThreads / 32 - 1) / (kPlanThreads / 32);
    if (ctas < by_seq) ctas = by_seq;
    if (ctas > kSmCount * 2) ctas = kSmCount * 2;
    unsigned char *const w = reinterpret_cast<unsigned char *>(ws);
    if (a.n_seq <= kPlanShared) {
        AWEQ_LAUNCH(kv_plan_kernel, dim3((unsigned)ctas), dim3(kPlanThreads), 0, stream, a, reinterpret_cast<unsigned *>(w));
        return AWEQ_OK;
    }
    PlanHead *const head = reinterpret_cast<PlanHead *>(w + kPlanHeadAt);
    PlanSeq *const seqs = reinterpret_cast<PlanSeq *>(w + kPlanSeqsAt);
    AWEQ_LAUNCH(kv_plan_sequences_kernel, dim3(1), dim3(kPlanThreads), 0, stream, a, head, seqs);
    AWEQ_LAUNCH(kv_plan_fill_kernel, dim3((unsigned)ctas), dim3(kPlanThreads), 0, stream, a, (const PlanHead *)head, (const PlanSeq *)seqs);
    return AWEQ_OK;
}

// ------------------------------------------------------------------ accept
// A CTA takes 128 16-byte pieces of a sequence's rows, a thread one piece of every row of the path, in the path's order.  Where the rows
// lie is looked up first, a thread per row.  Paths ascend, so a place is read before it is written (key path[j] = i is read for place
// j < i), whatever the piece: no thread needs another.  Bound by the chain of path, page, row: 8 sequences 5 us by itself, 256 (18 MB) 7.5.
constexpr int kAcceptThreads = 128;
__global__ void __launch_bounds__(kAcceptThreads) kv_accept_kernel(const KvAcceptArgs a, int pieces, int blocks)
{
    __shared__ long long from[kAcceptThreads], to[kAcceptThreads];
    __shared__ int first_bad, nodes[kAcceptThreads + 1];
    pdl_begin();
    const int tid = threadIdx.x, b = blockIdx.x / blocks, i = (blockIdx.x - b * blocks) * kAcceptThreads + tid;
    const bool lead = i == 0;
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
        if (key < 0 || key >= cap) return -1;
        const unsigned p = (unsigned)key / (unsigned)a.page_size;
        const int page = row[p];
        return page < 0 || page >= a.n_pages ? -1 : page * a.page_stride + (key - (long long)p * a.page_size) * a.token_stride;
    };
    if (tid == 0) nodes[0] = -1;
    for (int i0 = 0; i0 < n; i0 += kAcceptThreads) {
        const int count = min(n - i0, kAcceptThreads);
        if (tid == 0) first_bad = count;
        const int node = tid < count ? path[i0 + tid] : 0;
        if (tid < count) nodes[tid + 1] = node;
        __syncthreads();
        if (tid < count) {
            const long long x = place(base + node), y = place(base + i0 + tid);
            if (node <= nodes[tid] || x < 0 || y < 0) atomicMin(&first_bad, tid);
            from[tid] = x;
            to[tid] = node == i0 + tid ? -1 : y;
        }
        __syncthreads();
        // what comes before the first node that is out of order or nowhere
        const int good = first_bad;
        constexpr int U = 8;
        if (i < 2 * pieces)
            for (int j0 = 0; j0 < good; j0 += U) {
                uint4 x[U];
#pragma unroll
                for (int j = 0; j < U; ++j)
                    if (j0 + j < good && to[j0 + j] >= 0) x[j] = *reinterpret_cast<const uint4 *>(pool + from[j0 + j]);
#pragma unroll
                for (int j = 0; j < U; ++j)
                    if (j0 + j < good && to[j0 + j] >= 0) *reinterpret_cast<uint4 *>(pool + to[j0 + j]) = x[j];
            }
        if (good < count) {
            bad = true;
            break;
        }
        const int last = nodes[count];
        __syncthreads();
        if (tid == 0) nodes[0] = last;
    }
    if (lead && bad && a.st) atomicAdd(&a.st->out_of_range, 1ull);
}

aweq_status run_kv_accept(const KvAcceptArgs &a, cudaStream_t stream)
{
    const int pieces = a.n_kv * (a.head_dim / 8);
    const int blocks = (2 * pieces + kAcceptThreads - 1) / kAcceptThreads;
    AWEQ_LAUNCH(kv_accept_kernel, dim3((unsigned)(a.n_seq * blocks)), dim3(kAcceptThreads), 0, stream, a, pieces, blocks);
    return AWEQ_OK;
}

}  // namespace aweq
