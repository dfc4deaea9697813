// Bookkeeping of the cache's pages: one state of the sequences' tables into the next (fork, growth, fall back,
// end, copy on write), compaction, and the movement of the pages' data.  Whole numbers throughout; every result
// depends on the inputs alone: counts are integer atomics, and places in lists come from prefix sums.
//
// A plan is five small launches over arrays in the workspace:
//   clear    ref, grow and low of every page
//   count    a workgroup per slot: the pages it keeps (ref), and whether it grows into its last one (grow: how
//            many slots do, low: the lowest of them)
//   scan     which slots need copies and how many pages, as prefix sums over the slots; free pages per chunk
//   list     the free pages in order; page_ref and the counts
//   write    a workgroup per slot: its table row and its pair
// Compaction shares clear and count and has its own list and write.  The launches take 2 to 5 us each, so small tables are
// planned in one (a step of 64 slots with its two copies of pages: 14.0 us, with five launches 19.8; plans of 30000 entries: 22 and 20).
// The movement of data is bound by memory: 421 MB read and written in 71 us, 5.9 TB/s; compaction of 2.4 GB with its plan
// 437 us, 5.4 TB/s.
#include <limits.h>

#include <algorithm>

#include "kv_device.h"

namespace lora {

namespace {

constexpr int kThreads = 256;
constexpr int kChunk = 1024;              // pages of a workgroup in the lists
constexpr int kScanThreads = 1024;

// Workspace, in 32-bit words.
struct Ws {
    int32_t *ref, *grow, *low, *free, *chunk, *base, *cow, *head;   // head: flags, pages wanted, copies
};
enum { kHeadBad, kHeadWanted, kHeadMoves, kHeadWords = 64 };

__host__ __device__ inline int chunks_of(int n_pages) { return (n_pages + kChunk - 1) / kChunk; }

__host__ __device__ inline Ws ws_of(int32_t *w, int n_pages, int n_seqs)
{
    Ws s;
    s.head = w;
    s.ref = w + kHeadWords;
    s.grow = s.ref + n_pages;
    s.low = s.grow + n_pages;
    s.free = s.low + n_pages;
    s.chunk = s.free + n_pages;
    s.base = s.chunk + chunks_of(n_pages);
    s.cow = s.base + n_seqs;
    return s;
}

__device__ inline int pages_of(int tokens, int shift) { return (int)(((int64_t)tokens + (1 << shift) - 1) >> shift); }

// What slot s of the next state keeps: the slot it comes from (-1: none), tokens kept and its new length.
struct Slot {
    int src, keep, len;
};

__device__ inline Slot slot_of(const PlanParams &p, int s, unsigned &bad)
{
    Slot r;
    r.src = p.src ? p.src[s] : s;
    if (r.src < -1 || r.src >= p.n_seqs) bad |= LORA_STATUS_BAD_SEQ, r.src = -1;
    const int64_t room = (int64_t)p.max_pages << p.page_shift;
    int had = r.src < 0 ? 0 : p.from_len[r.src];
    r.len = p.new_len ? p.new_len[s] : had;
    if (had < 0 || had > room) bad |= LORA_STATUS_BAD_LENGTH, had = 0;
    if (r.len < 0 || r.len > room) bad |= LORA_STATUS_BAD_LENGTH, r.len = 0;
    r.keep = min(had, r.len);
    return r;
}

__device__ inline bool grows(const PlanParams &p, const Slot &r)
{
    return r.len > r.keep && (r.keep & ((1 << p.page_shift) - 1)) != 0;
}

__global__ __launch_bounds__(kThreads) void clear_kernel(PlanParams p)
{
    const Ws w = ws_of(p.ws, p.n_pages, p.n_seqs);
    const int i = blockIdx.x * kThreads + threadIdx.x;
    if (i < kHeadWords) w.head[i] = 0;
    if (i < p.n_pages) {
        w.ref[i] = 0;
        w.grow[i] = 0;
        w.low[i] = INT_MAX;
    }
}

__global__ __launch_bounds__(kThreads) void count_kernel(PlanParams p)
{
    const Ws w = ws_of(p.ws, p.n_pages, p.n_seqs);
    const int s = blockIdx.x;
    unsigned bad = 0;
    const Slot r = slot_of(p, s, bad);
    const int kept = pages_of(r.keep, p.page_shift);
    const int32_t *row = p.from_table + (int64_t)max(r.src, 0) * p.max_pages;
    for (int i = threadIdx.x; i < kept; i += kThreads) {
        const int page = row[i];
        if ((unsigned)page >= (unsigned)p.n_pages) {
            bad |= LORA_STATUS_BAD_PAGE;
            continue;
        }
        atomicAdd(&w.ref[page], 1);
        if (i == kept - 1 && grows(p, r)) {
            atomicAdd(&w.grow[page], 1);
            atomicMin(&w.low[page], s);
        }
    }
    if (bad) atomicOr((unsigned *)&w.head[kHeadBad], bad);
}

// Copies of a page that the plan asks for: every slot that grows into a page it shares writes to one of its
// own, but the lowest one keeps it where nobody else reads on.
__device__ inline int copies_of(int ref, int grow)
{
    return ref <= 1 ? 0 : grow == ref ? grow - 1 : grow;
}

// Workgroup b < chunks: free pages of a chunk.  The last workgroup: the slots' needs.
__global__ __launch_bounds__(kScanThreads) void scan_kernel(PlanParams p)
{
    const Ws w = ws_of(p.ws, p.n_pages, p.n_seqs);
    const int chunks = chunks_of(p.n_pages);
    const int tid = threadIdx.x;
    int total;
    if ((int)blockIdx.x < chunks) {
        const int page = blockIdx.x * kChunk + tid;
        block_scan<kScanThreads / 64>((int)(page < p.n_pages && w.ref[page] == 0), total);
        if (tid == 0) w.chunk[blockIdx.x] = total;
        return;
    }
    if (w.head[kHeadBad]) return;         // the pages looked up below would not all be pages
    int64_t wanted = 0;                   // a plan may ask for more pages than an int holds
    int copies = 0;
    for (int s0 = 0; s0 < p.n_seqs; s0 += kScanThreads) {
        const int s = s0 + tid;
        int need = 0, cow = 0;
        if (s < p.n_seqs) {
            unsigned bad = 0;
            const Slot r = slot_of(p, s, bad);
            const int kept = pages_of(r.keep, p.page_shift);
            if (grows(p, r)) {
                const int page = p.from_table[(int64_t)r.src * p.max_pages + kept - 1];
                const int ref = w.ref[page];
                cow = ref > 1 && !(w.grow[page] == ref && w.low[page] == s);
            }
            need = cow + pages_of(r.len, p.page_shift) - kept;
        }
        int64_t sum_need;
        int sum_cow;
        const int64_t at = block_scan<kScanThreads / 64>((int64_t)need, sum_need);
        const int cow_at = block_scan<kScanThreads / 64>(cow, sum_cow);
        if (s < p.n_seqs) {
            w.base[s] = (int)(wanted + at - need);
            w.cow[s] = cow ? copies + cow_at - 1 : -1;
        }
        wanted += sum_need;
        copies += sum_cow;
    }
    if (tid == 0) {
        w.head[kHeadWanted] = (int)min(wanted, (int64_t)INT_MAX);
        w.head[kHeadMoves] = copies;
    }
}

// Sum of chunk[0 .. b) and of all chunks, for a workgroup of kScanThreads.
__device__ inline int chunks_before(const Ws &w, int chunks, int b, int &all)
{
    int before = 0, sum = 0;
    for (int i = threadIdx.x; i < chunks; i += kScanThreads) {
        sum += w.chunk[i];
        before += i < b ? w.chunk[i] : 0;
    }
    int total;
    block_scan<kScanThreads / 64>(before, total);
    before = total;
    block_scan<kScanThreads / 64>(sum, all);
    return before;
}

__global__ __launch_bounds__(kScanThreads) void list_kernel(PlanParams p)
{
    const Ws w = ws_of(p.ws, p.n_pages, p.n_seqs);
    int n_free, dummy;
    const int before = chunks_before(w, chunks_of(p.n_pages), blockIdx.x, n_free);
    const int page = blockIdx.x * kChunk + threadIdx.x;
    const bool inside = page < p.n_pages;
    const int ref = inside ? w.ref[page] : 1;
    const int rank = before + block_scan<kScanThreads / 64>((int)(ref == 0), dummy) - 1;
    const unsigned bad = w.head[kHeadBad];
    const int wanted = w.head[kHeadWanted];
    const bool go = !bad && wanted <= n_free;
    if (inside && ref == 0) w.free[rank] = page;
    if (inside && p.to_ref) {
        if (go) p.to_ref[page] = ref ? ref - copies_of(ref, w.grow[page]) : rank < wanted;
        else if (p.from_ref) p.to_ref[page] = p.from_ref[page];
    }
    if (blockIdx.x == 0 && threadIdx.x == 0) {
        const int used = p.n_pages - n_free + (go ? wanted : 0);
        p.counts[0] = go ? used : 0;
        p.counts[1] = go ? w.head[kHeadMoves] : 0;
        p.counts[2] = go ? p.n_pages - used : 0;
        p.counts[3] = bad ? 0 : wanted;
        if (!go) atomicOr(p.status, bad ? bad : (unsigned)LORA_STATUS_NO_PAGES);
    }
}

__global__ __launch_bounds__(kThreads) void write_kernel(PlanParams p)
{
    const Ws w = ws_of(p.ws, p.n_pages, p.n_seqs);
    const int s = blockIdx.x;
    int n_free = 0;
    for (int i = threadIdx.x; i < chunks_of(p.n_pages); i += kThreads) n_free += w.chunk[i];
    int total;
    block_scan<kThreads / 64>(n_free, total);
    int32_t *to = p.to_table + (int64_t)s * p.max_pages;
    if (w.head[kHeadBad] || w.head[kHeadWanted] > total) {
        const int32_t *from = p.from_table + (int64_t)s * p.max_pages;
        for (int i = threadIdx.x; i < p.max_pages; i += kThreads) to[i] = from[i];
        if (threadIdx.x == 0) p.to_len[s] = p.from_len[s];
        return;
    }
    unsigned bad = 0;
    const Slot r = slot_of(p, s, bad);
    const int kept = pages_of(r.keep, p.page_shift), now = pages_of(r.len, p.page_shift);
    const int32_t *from = p.from_table + (int64_t)max(r.src, 0) * p.max_pages;
    const int base = w.base[s], move = w.cow[s];
    const int grown = base + (move >= 0);
    for (int i = threadIdx.x; i < p.max_pages; i += kThreads) {
        int page = -1;
        if (i < kept) {
            page = from[i];
            if (move >= 0 && i == kept - 1) {
                const int mine = w.free[base];
                p.pairs[2 * move] = page;
                p.pairs[2 * move + 1] = mine;
                page = mine;
            }
        } else if (i < now) {
            page = w.free[grown + i - kept];
        }
        to[i] = page;
    }
    if (threadIdx.x == 0) p.to_len[s] = r.len;
}

// ---- a plan in one launch, for caches of up to kSmallPages pages (what LDS holds) and tables of up to kSmallTable entries (beyond
// it, one CU's share of the loads costs more than the launches): one workgroup does
// the steps above with its arrays in LDS.  Waves take slots in turn, with the table entries of eight slots on their way at a time. ----

constexpr int kSmallPages = 8192, kSmallSeqs = 1024, kSmallTable = 1 << 14;
constexpr int kDeep = 8;

__global__ __launch_bounds__(kScanThreads) void small_plan_kernel(PlanParams p)
{
    __shared__ int s_ref[kSmallPages], s_grow[kSmallPages], s_low[kSmallPages], s_free[kSmallPages];
    __shared__ int s_src[kSmallSeqs], s_keep[kSmallSeqs], s_len[kSmallSeqs];     // then: pages kept and asked for
    constexpr int WAVES = kScanThreads / 64;
    __shared__ int s_base[kSmallSeqs], s_cow[kSmallSeqs], s_sum[2][WAVES];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    for (int i = tid; i < p.n_pages; i += kScanThreads) {
        s_ref[i] = 0;
        s_grow[i] = 0;
        s_low[i] = INT_MAX;
    }
    unsigned bad = 0;
    Slot own = {-1, 0, 0};
    if (tid < p.n_seqs) {
        own = slot_of(p, tid, bad);
        s_src[tid] = max(own.src, 0);
        s_keep[tid] = pages_of(own.keep, p.page_shift);
        s_len[tid] = pages_of(own.len, p.page_shift);
        s_cow[tid] = grows(p, own);
    }
    __syncthreads();
    int most = 0;                         // of the slots' table entries in use, now and then
    for (int s = lane; s < p.n_seqs; s += 64) most = max(most, max(s_keep[s], s_len[s]));
#pragma unroll
    for (int d = 32; d; d >>= 1) most = max(most, __shfl_xor(most, d));
    for (int s0 = wave; s0 < p.n_seqs; s0 += WAVES * kDeep) {
        int keep[kDeep];
        const int32_t *row[kDeep];
        const int mine = min(s0 + (lane & (kDeep - 1)) * WAVES, p.n_seqs - 1);       // lane k looks up slot k of the eight
        const int my_keep = s_keep[mine], my_src = s_src[mine];
#pragma unroll
        for (int k = 0; k < kDeep; ++k) {
            keep[k] = s0 + k * WAVES < p.n_seqs ? __builtin_amdgcn_readlane(my_keep, k) : 0;
            row[k] = p.from_table + (int64_t)__builtin_amdgcn_readlane(my_src, k) * p.max_pages;
        }
        for (int i0 = 0; i0 < most; i0 += 64) {
            const int i = i0 + lane;
            int page[kDeep];
#pragma unroll
            for (int k = 0; k < kDeep; ++k) page[k] = row[k][min(i, p.max_pages - 1)];
#pragma unroll
            for (int k = 0; k < kDeep; ++k) {
                if (i >= keep[k]) continue;
                if ((unsigned)page[k] >= (unsigned)p.n_pages) {
                    bad |= LORA_STATUS_BAD_PAGE;
                    continue;
                }
                atomicAdd(&s_ref[page[k]], 1);
                if (i == keep[k] - 1) {
                    const int s = s0 + k * WAVES;
                    s_base[s] = page[k];  // the last page, until the base takes its place
                    if (s_cow[s]) {
                        atomicAdd(&s_grow[page[k]], 1);
                        atomicMin(&s_low[page[k]], s);
                    }
                }
            }
        }
    }
    __shared__ unsigned s_bad;
    if (tid == 0) s_bad = 0;
    __syncthreads();
    if (bad) atomicOr(&s_bad, bad);
    __syncthreads();
    bad = s_bad;
    int wanted = 0, copies = 0, n_free = 0;
    if (!bad) {
        int need = 0, cow = 0;
        if (tid < p.n_seqs) {
            if (s_cow[tid]) {
                const int page = s_base[tid], ref = s_ref[page];
                cow = ref > 1 && !(s_grow[page] == ref && s_low[page] == tid);
            }
            need = cow + s_len[tid] - s_keep[tid];
        }
        // a thread looks at eight pages that lie together
        int free = 0;
#pragma unroll
        for (int k = 0; k < kSmallPages / kScanThreads; ++k) {
            const int i = tid * (kSmallPages / kScanThreads) + k;
            free += i < p.n_pages && s_ref[i] == 0;
        }
        // pages asked for and copies in one number: no more than kSmallTable + kSmallSeqs and kSmallSeqs in all
        const int both = need << 11 | cow, upto = wave_scan(both), upto_free = wave_scan(free);
        static_assert(((int64_t)kSmallTable + kSmallSeqs) << 11 < INT_MAX && kSmallSeqs < 1 << 11, "both fit");
        if (lane == 63) s_sum[0][wave] = upto, s_sum[1][wave] = upto_free;
        __syncthreads();
        int before = upto - both, rank = upto_free - free, total = 0;
#pragma unroll
        for (int w = 0; w < WAVES; ++w) {
            if (w < wave) before += s_sum[0][w], rank += s_sum[1][w];
            total += s_sum[0][w];
            n_free += s_sum[1][w];
        }
        wanted = total >> 11;
        copies = total & 2047;
        if (tid < p.n_seqs) {
            s_base[tid] = before >> 11;
            s_cow[tid] = cow ? before & 2047 : -1;
        }
#pragma unroll
        for (int k = 0; k < kSmallPages / kScanThreads; ++k) {
            const int i = tid * (kSmallPages / kScanThreads) + k;
            if (i >= p.n_pages || s_ref[i]) continue;
            s_free[rank] = i;
            s_low[i] = rank++;            // of a free page
        }
        __syncthreads();
    }
    const bool go = !bad && wanted <= n_free;
    if (p.to_ref)
        for (int i = tid; i < p.n_pages; i += kScanThreads) {
            if (go) p.to_ref[i] = s_ref[i] ? s_ref[i] - copies_of(s_ref[i], s_grow[i]) : s_low[i] < wanted;
            else if (p.from_ref) p.to_ref[i] = p.from_ref[i];
        }
    if (tid == 0) {
        const int used = p.n_pages - n_free + (go ? wanted : 0);
        p.counts[0] = go ? used : 0;
        p.counts[1] = go ? copies : 0;
        p.counts[2] = go ? p.n_pages - used : 0;
        p.counts[3] = bad ? 0 : wanted;
        if (!go) atomicOr(p.status, bad ? bad : (unsigned)LORA_STATUS_NO_PAGES);
    }
    if (tid < p.n_seqs) p.to_len[tid] = go ? own.len : p.from_len[tid];
    for (int s0 = wave; s0 < p.n_seqs; s0 += WAVES * kDeep) {
        int keep[kDeep], now[kDeep], base[kDeep], move[kDeep];
        const int32_t *row[kDeep];
        const int mine = min(s0 + (lane & (kDeep - 1)) * WAVES, p.n_seqs - 1);
        const int my_keep = go ? s_keep[mine] : p.max_pages, my_len = go ? s_len[mine] : p.max_pages, my_base = go ? s_base[mine] : 0;
        const int my_move = go ? s_cow[mine] : -1, my_src = go ? s_src[mine] : mine;
#pragma unroll
        for (int k = 0; k < kDeep; ++k) {
            keep[k] = __builtin_amdgcn_readlane(my_keep, k);
            now[k] = __builtin_amdgcn_readlane(my_len, k);
            base[k] = __builtin_amdgcn_readlane(my_base, k);
            move[k] = __builtin_amdgcn_readlane(my_move, k);
            row[k] = p.from_table + (int64_t)__builtin_amdgcn_readlane(my_src, k) * p.max_pages;
        }
        for (int i0 = 0; i0 < p.max_pages; i0 += 64) {
            const int i = i0 + lane;
            int page[kDeep];
#pragma unroll
            for (int k = 0; k < kDeep; ++k) page[k] = row[k][min(i, p.max_pages - 1)];
#pragma unroll
            for (int k = 0; k < kDeep; ++k) {
                const int s = s0 + k * WAVES;
                if (s >= p.n_seqs || i >= p.max_pages) continue;
                if (move[k] >= 0 && i == keep[k] - 1) {
                    p.pairs[2 * move[k]] = page[k];
                    p.pairs[2 * move[k] + 1] = page[k] = s_free[base[k]];
                } else if (i >= keep[k]) {
                    page[k] = i < now[k] ? s_free[base[k] + (move[k] >= 0) + i - keep[k]] : -1;
                }
                p.to_table[(int64_t)s * p.max_pages + i] = page[k];
            }
        }
    }
}

// ---- compaction: pages in use with numbers from the number of pages in use on move to the free numbers below.
// The r-th such page, in order, goes to the r-th free number.  chunk holds free pages per chunk, as above. ----

// Free pages among the numbers below n.
__device__ inline int free_below(const Ws &w, int n)
{
    const int full = n / kChunk;
    int sum = 0;
    for (int i = threadIdx.x; i < full; i += kScanThreads) sum += w.chunk[i];
    const int page = full * kChunk + (int)threadIdx.x;
    if (page < n) sum += w.ref[page] == 0;
    int total;
    block_scan<kScanThreads / 64>(sum, total);
    return total;
}

__global__ __launch_bounds__(kScanThreads) void compact_list_kernel(PlanParams p)
{
    const Ws w = ws_of(p.ws, p.n_pages, p.n_seqs);
    int n_free, dummy;
    const int before = chunks_before(w, chunks_of(p.n_pages), blockIdx.x, n_free);
    const unsigned bad = w.head[kHeadBad];
    const int live = p.n_pages - n_free;
    const int holes = free_below(w, live);                 // as many as pages that move
    const int page = blockIdx.x * kChunk + threadIdx.x;
    const bool inside = page < p.n_pages;
    const int ref = inside ? w.ref[page] : 1;
    const int free_rank = before + block_scan<kScanThreads / 64>((int)(ref == 0), dummy) - (ref == 0);   // free numbers below `page`
    if (inside && !bad) {
        // pages in use among the numbers from `live` to `page`: those below `page` less those below `live`
        const int mover = page - free_rank - (live - holes);
        if (ref == 0 && page < live) p.pairs[2 * free_rank + 1] = page;
        if (ref != 0 && page >= live) {
            p.pairs[2 * mover] = page;
            w.low[page] = mover;
        }
        if (page >= live && p.to_ref) p.to_ref[page] = 0;
    }
    if (inside && bad && p.to_ref && p.from_ref) p.to_ref[page] = p.from_ref[page];
    if (blockIdx.x == 0 && threadIdx.x == 0) {
        p.counts[0] = bad ? 0 : live;
        p.counts[1] = bad ? 0 : holes;
        p.counts[2] = bad ? 0 : n_free;
        p.counts[3] = 0;
        if (bad) atomicOr(p.status, bad);
        w.head[kHeadWanted] = live;
    }
}

// Workgroups from n_seqs on carry page_ref over.
__global__ __launch_bounds__(kThreads) void compact_write_kernel(PlanParams p)
{
    const Ws w = ws_of(p.ws, p.n_pages, p.n_seqs);
    const bool bad = w.head[kHeadBad] != 0;
    const int live = w.head[kHeadWanted];
    if ((int)blockIdx.x >= p.n_seqs) {
        const int page = (blockIdx.x - p.n_seqs) * kThreads + threadIdx.x;
        if (bad || page >= p.n_pages) return;
        const int ref = w.ref[page];
        if (ref) p.to_ref[page < live ? page : p.pairs[2 * w.low[page] + 1]] = ref;
        return;
    }
    const int s = blockIdx.x;
    const int len = p.from_len[s];
    const int held = bad ? p.max_pages : pages_of(len, p.page_shift);
    const int32_t *from = p.from_table + (int64_t)s * p.max_pages;
    int32_t *to = p.to_table + (int64_t)s * p.max_pages;
    for (int i = threadIdx.x; i < p.max_pages; i += kThreads) {
        int page = -1;
        if (i < held) {
            page = from[i];
            if (!bad && page >= live) page = p.pairs[2 * w.low[page] + 1];
        }
        to[i] = page;
    }
    if (threadIdx.x == 0) p.to_len[s] = len;
}

// ---- data ----

constexpr int kCopyVecs = 4;                           // 16-byte pieces of a thread

__global__ __launch_bounds__(kThreads) void copy_kernel(CopyParams p)
{
    const int n = min(min(p.counts[1], p.max_moves), p.n_pages);
    const int layer = blockIdx.z >> 1;
    uint16_t *base = ((blockIdx.z & 1) ? p.v : p.k) + layer * p.layer_stride;
    const int vecs = p.outer * p.inner * (p.run >> 3);
    for (int m = blockIdx.y; m < n; m += gridDim.y) {
        const int from = p.pairs[2 * m], to = p.pairs[2 * m + 1];
        if ((unsigned)from >= (unsigned)p.n_pages || (unsigned)to >= (unsigned)p.n_pages) continue;
        const uint16_t *src = base + from * p.page_stride;
        uint16_t *dst = base + to * p.page_stride;
        u32x4 x[kCopyVecs];
        int64_t at[kCopyVecs];
#pragma unroll
        for (int j = 0; j < kCopyVecs; ++j) {
            const int i = blockIdx.x * kThreads * kCopyVecs + j * kThreads + threadIdx.x;
            const int r = i / p.run_vecs, e = i - r * (p.run >> 3);
            const int o = r / p.inner_div, k = r - o * p.inner;
            at[j] = i < vecs ? o * p.outer_stride + k * p.inner_stride + 8 * e : -1;
            if (at[j] >= 0) x[j] = ld16<true>(src + at[j]);
        }
#pragma unroll
        for (int j = 0; j < kCopyVecs; ++j)
            if (at[j] >= 0) st16<true>(dst + at[j], x[j]);
    }
}

}  // namespace

size_t plan_ws_bytes(int n_pages, int n_seqs)
{
    return ((size_t)kHeadWords + 4 * (size_t)n_pages + chunks_of(n_pages) + 2 * (size_t)n_seqs) * sizeof(int32_t);
}

hipError_t launch_plan(const PlanParams &p, hipStream_t s)
{
    if (p.n_pages <= kSmallPages && p.n_seqs <= kSmallSeqs && (int64_t)p.n_seqs * p.max_pages <= kSmallTable) {
        hipLaunchKernelGGL(small_plan_kernel, dim3(1), dim3(kScanThreads), 0, s, p);
        return hipGetLastError();
    }
    const int chunks = chunks_of(p.n_pages);
    hipLaunchKernelGGL(clear_kernel, dim3((std::max(p.n_pages, (int)kHeadWords) + kThreads - 1) / kThreads), dim3(kThreads), 0, s, p);
    hipLaunchKernelGGL(count_kernel, dim3(p.n_seqs), dim3(kThreads), 0, s, p);
    hipLaunchKernelGGL(scan_kernel, dim3(chunks + 1), dim3(kScanThreads), 0, s, p);
    hipLaunchKernelGGL(list_kernel, dim3(chunks), dim3(kScanThreads), 0, s, p);
    hipLaunchKernelGGL(write_kernel, dim3(p.n_seqs), dim3(kThreads), 0, s, p);
    return hipGetLastError();
}

hipError_t launch_compact(const PlanParams &p, hipStream_t s)
{
    const int chunks = chunks_of(p.n_pages);
    hipLaunchKernelGGL(clear_kernel, dim3((std::max(p.n_pages, (int)kHeadWords) + kThreads - 1) / kThreads), dim3(kThreads), 0, s, p);
    hipLaunchKernelGGL(count_kernel, dim3(p.n_seqs), dim3(kThreads), 0, s, p);
    hipLaunchKernelGGL(scan_kernel, dim3(chunks + 1), dim3(kScanThreads), 0, s, p);
    hipLaunchKernelGGL(compact_list_kernel, dim3(chunks), dim3(kScanThreads), 0, s, p);
    const int extra = p.to_ref ? (p.n_pages + kThreads - 1) / kThreads : 0;
    hipLaunchKernelGGL(compact_write_kernel, dim3(p.n_seqs + extra), dim3(kThreads), 0, s, p);
    return hipGetLastError();
}

hipError_t launch_copy_pages(const CopyParams &p, hipStream_t s)
{
    const int vecs = p.outer * p.inner * (p.run >> 3);
    const int per = kThreads * kCopyVecs;
    const dim3 grid((vecs + per - 1) / per, std::min(p.max_moves, 4096), 2 * p.n_layers);
    hipLaunchKernelGGL(copy_kernel, grid, dim3(kThreads), 0, s, p);
    return hipGetLastError();
}

}  // namespace lora
