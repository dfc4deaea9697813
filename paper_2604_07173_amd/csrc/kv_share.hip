// Which sequences of a batch hold the same first pages.  Whole numbers throughout; every result depends on the inputs alone: places
// come from prefix sums, and the atomics are sums, minima and a hash table whose slots' numbers nobody sees.
//
//   lead     a sequence's leader: the lowest one with the same page at place min_pages - 1, found through a hash table of page numbers
//   common   a wave per sequence: table entries that agree with the leader's, 256 at a time; members, least agreement and rows of each leader
//   place    groups numbered by their leaders; their rows listed one group after another, members in order
//
// Bound by latency: a chain of loads, atomics and barriers (the entries to compare are a few hundred bytes a sequence).  Batches with
// few entries take one launch, in LDS; a wave compares one sequence after another there, so larger ones take three.
#include <limits.h>

#include <algorithm>

#include "kv_device.h"
#include "kv_work.h"

namespace lora {

namespace {

constexpr int kThreads = 1024, kWaves = kThreads / 64;
constexpr int kSeqsInLds = 1024;          // sequences whose arrays fit in LDS
constexpr int kWide = 4;                  // entries of a table that a lane compares at a time
// Rounds of comparing that the waves of one workgroup take on, at most: sequences x their rounds (of one round each, in one launch and in
// three: 4 sequences 7.8 and 12.5 us, 32 10.3 and 13.1, 64 11.5 and 13.4, 128 16.9 and 13.8, 256 28.3 and 14.8).
constexpr int kOneLaunch = 5 * kWaves;

typedef unsigned long long u64;

// Arrays over the hash table's slots, then over the sequences.
struct Arrays {
    u64 *key;                             // 2^32 + the page, 0 = none
    int32_t *first;                       // lowest sequence with that page
    int32_t *slot, *lead, *common, *members, *least, *total, *next;
};
constexpr int kSeqArraysShare = 7;

__host__ __device__ inline int hash_size(int n)
{
    int h = 64;
    while (h < 2 * n) h *= 2;
    return h;
}

__host__ __device__ inline size_t words_of(int n) { return 3 * (size_t)hash_size(n) + kSeqArraysShare * (size_t)n; }

__device__ inline Arrays arrays_of(int32_t *w, int n)
{
    Arrays a;
    const int h = hash_size(n);
    a.key = reinterpret_cast<u64 *>(w);
    a.first = w + 2 * (size_t)h;
    a.slot = a.first + h;
    a.lead = a.slot + n;
    a.common = a.lead + n;
    a.members = a.common + n;
    a.least = a.members + n;
    a.total = a.least + n;
    a.next = a.total + n;
    return a;
}

// What atomics of this workgroup or of a launch before have left: past the CU's own cache.
__device__ inline int32_t fresh(const int32_t *p) { return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }

struct Seq {
    int rows, whole;                      // new rows, whole pages before the first of them
    bool part;                            // it may share
    unsigned bad;                         // as faults_of in kv_attention.h
};

__device__ inline Seq seq_of(const ShareParams &p, int s)
{
    const int first = p.b.row_start[s], end = p.b.row_start[s + 1], len = p.b.seq_len[s];
    Seq q;
    q.bad = len < 0 || len > p.b.tokens_max;
    if (first < 0 || end < first || end > p.b.n_rows || (s == 0 && first != 0) || (s == p.b.n_seqs - 1 && end != p.b.n_rows)) q.bad |= 2;
    q.rows = q.bad & 2 ? 0 : end - first;
    q.whole = q.bad ? 0 : max(0, len - q.rows) >> p.page_shift;
    q.part = !q.bad && q.rows >= 1 && q.rows <= p.max_rows && q.whole >= p.min_pages;
    return q;
}

__device__ inline void find_leaders(const ShareParams &p, const Arrays &a)
{
    const int n = p.b.n_seqs, h = hash_size(n);
    unsigned bad = 0;
    for (int i = threadIdx.x; i < h; i += kThreads) {
        a.key[i] = 0;
        a.first[i] = INT_MAX;
    }
    for (int s = threadIdx.x; s < n; s += kThreads) bad |= seq_of(p, s).bad;
    if (bad) atomicOr(p.b.status, LORA_STATUS_BAD_LENGTH);
    const bool none = __syncthreads_or(bad & 2);      // rows that are no partition: no groups
    for (int s = threadIdx.x; s < n; s += kThreads) {
        a.members[s] = 0;
        a.least[s] = INT_MAX;
        a.total[s] = 0;
        int at = -1;
        if (!none && seq_of(p, s).part) {
            const u64 key = (u64)1 << 32 | (unsigned)p.b.table[(int64_t)s * p.b.max_pages + p.min_pages - 1];
            // at most n of the h >= 2 n slots are ever taken, so a free one or the key's own is found
            for (at = (int)(((unsigned)key * 2654435769u) >> 7) & (h - 1);; at = (at + 1) & (h - 1)) {
                const u64 was = atomicCAS(&a.key[at], 0ull, key);
                if (was == 0 || was == key) break;
            }
            atomicMin(&a.first[at], s);
        }
        a.slot[s] = at;
    }
    __syncthreads();
    for (int s = threadIdx.x; s < n; s += kThreads) a.lead[s] = a.slot[s] < 0 ? -1 : fresh(&a.first[a.slot[s]]);
}

// Leading table entries of the sequences s, s + stride .. (N of them) that agree with their leaders', by a wave: of all of them at once,
// as a comparison is little but the latency of its loads.
template <int N>
__device__ inline void compare(const ShareParams &p, const Arrays &a, int s0, int stride)
{
    const int lane = threadIdx.x & 63, n = p.b.n_seqs;
    int lead[N], common[N], rows[N];
#pragma unroll
    for (int k = 0; k < N; ++k) lead[k] = s0 + k * stride < n ? uniform(a.lead[s0 + k * stride]) : -1;
    int most = 0;
#pragma unroll
    for (int k = 0; k < N; ++k) {
        const Seq q = seq_of(p, lead[k] < 0 ? 0 : s0 + k * stride), l = seq_of(p, max(lead[k], 0));
        common[k] = lead[k] < 0 ? 0 : uniform(min(q.whole, l.whole));
        rows[k] = q.rows;
        if (lead[k] != s0 + k * stride) most = max(most, common[k]);
    }
    for (int at = 0; at < most; at += 64 * kWide) {
        int x[N][kWide], y[N][kWide];
#pragma unroll
        for (int k = 0; k < N; ++k) {
            const int64_t mine = (int64_t)min(s0 + k * stride, n - 1) * p.b.max_pages, its = (int64_t)max(lead[k], 0) * p.b.max_pages;
#pragma unroll
            for (int w = 0; w < kWide; ++w) {
                const int i = max(0, min(at + w * 64 + lane, common[k] - 1));
                x[k][w] = p.b.table[mine + i];
                y[k][w] = p.b.table[its + i];
            }
        }
        most = 0;
#pragma unroll
        for (int k = 0; k < N; ++k) {
            if (lead[k] < 0 || lead[k] == s0 + k * stride || at >= common[k]) continue;
            int differ = INT_MAX;
#pragma unroll
            for (int w = kWide - 1; w >= 0; --w) {
                const u64 mask = __ballot(x[k][w] != y[k][w]);
                if (mask) differ = at + w * 64 + __ffsll(mask) - 1;
            }
            common[k] = min(common[k], differ);           // below `at` + 256 then, which ends it
            most = max(most, common[k]);
        }
    }
#pragma unroll
    for (int k = 0; k < N; ++k) {
        const int s = s0 + k * stride;
        if (lane != 0 || s >= n) continue;
        a.common[s] = common[k];
        if (lead[k] < 0 || common[k] < p.min_pages) continue;
        atomicAdd(&a.members[lead[k]], 1);
        atomicMin(&a.least[lead[k]], common[k]);
        atomicAdd(&a.total[lead[k]], rows[k]);
    }
}

__device__ inline void list_groups(const ShareParams &p, const Arrays &a)
{
    __shared__ u64 s_spared;
    const int n = p.b.n_seqs, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    // groups, members and rows in one number: 21 bits each are enough for 2^20
    constexpr int MEMBERS = 21, ROWS = 42;
    constexpr u64 MASK = ((u64)1 << 21) - 1;
    u64 sums = 0;
    if (tid == 0) s_spared = 0;
    for (int s0 = 0; s0 < n; s0 += kThreads) {
        const int s = s0 + tid;
        int members = 0, total = 0, least = 0;
        if (s < n && a.lead[s] == s) {
            members = fresh(&a.members[s]);
            total = fresh(&a.total[s]);
            least = fresh(&a.least[s]);
        }
        const bool head = members >= 2;
        const u64 own = head ? 1 | (u64)members << MEMBERS | (u64)total << ROWS : 0;
        u64 all;
        const u64 before = sums + block_scan<kWaves>(own, all) - own;
        if (head) {
            int32_t *g = p.groups + 4 * (int64_t)(before & MASK);
            g[0] = s;
            g[1] = least << p.page_shift;
            g[2] = (int)(before >> ROWS);
            g[3] = total;
            a.next[s] = (int)(before >> ROWS);
            atomicAdd(&s_spared, (u64)(members - 1) * ((u64)least << p.page_shift));
        }
        sums += all;
    }
    __syncthreads();
    const int groups = (int)(sums & MASK), rows = (int)(sums >> ROWS);
    if (tid == 0) {
        p.counts[0] = groups;
        p.counts[1] = rows;
        p.counts[2] = (int)(sums >> MEMBERS & MASK);
        p.counts[3] = (int32_t)min(s_spared, (u64)INT_MAX);
    }
    for (int64_t i = 4 * (int64_t)groups + tid; i < 4 * (int64_t)p.most; i += kThreads) p.groups[i] = i & 3 ? 0 : -1;
    for (int i = rows + tid; i < p.most_rows; i += kThreads) p.rows[i] = -1;
    for (int s0 = 0; s0 < n; s0 += kThreads) {
        const int s = s0 + tid;
        int lead = s < n ? a.lead[s] : -1;
        if (lead >= 0 && (a.common[s] < p.min_pages || fresh(&a.members[lead]) < 2)) lead = -1;
        const Seq q = lead >= 0 ? seq_of(p, s) : Seq{};
        // the wave's members of the same group, as lanes: those that agree with this one in every bit of the leader's number; and their
        // rows, bit by bit: those before this one, and all
        u64 same = __ballot(lead >= 0);
        for (int bit = 0; (n - 1) >> bit; ++bit) {
            const u64 set = __ballot(lead >> bit & 1);
            same &= lead >> bit & 1 ? set : ~set;
        }
        int before = 0, all = 0;
        for (int bit = 0; __any(q.rows >> bit); ++bit) {
            const u64 set = __ballot(q.rows >> bit & 1) & same;
            before += __popcll(set & (((u64)1 << lane) - 1)) << bit;
            all += __popcll(set) << bit;
        }
        const bool last = lead >= 0 && same >> lane == 1;
        // one wave after another takes its part of every group's rows
        int at = -1;
        const int waves = min(kWaves, (n - s0 + 63) >> 6);
        for (int w = 0; w < waves; ++w) {
            if (w == wave && lead >= 0) {
                const int base = a.next[lead];
                at = base + before;
                if (last) a.next[lead] = base + all;
            }
            __syncthreads();
        }
        if (s < n) {
            p.own[s] = lead < 0 ? 0 : fresh(&a.least[lead]) << p.page_shift;
            p.place[s] = at;
            const int row0 = lead < 0 ? 0 : p.b.row_start[s];
            for (int i = 0; i < q.rows; ++i) p.rows[at + i] = row0 + i;
        }
    }
}

__global__ __launch_bounds__(kThreads) void share_kernel(ShareParams p)
{
    constexpr int WORDS = 3 * 2 * kSeqsInLds + kSeqArraysShare * kSeqsInLds;
    __shared__ __align__(16) int32_t s_mem[WORDS];
    const Arrays a = arrays_of(s_mem, p.b.n_seqs);
    find_leaders(p, a);
    __syncthreads();
    for (int s = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6); s < p.b.n_seqs; s += 4 * kWaves) compare<4>(p, a, s, kWaves);
    __syncthreads();
    list_groups(p, a);
}

__global__ __launch_bounds__(kThreads) void lead_kernel(ShareParams p) { find_leaders(p, arrays_of(p.ws, p.b.n_seqs)); }

__global__ __launch_bounds__(256) void common_kernel(ShareParams p)
{
    const Arrays a = arrays_of(p.ws, p.b.n_seqs);
    const int s = __builtin_amdgcn_readfirstlane(blockIdx.x * 4 + (threadIdx.x >> 6));
    if (s < p.b.n_seqs) compare<1>(p, a, s, 1);
}

__global__ __launch_bounds__(kThreads) void place_kernel(ShareParams p)
{
    __shared__ int32_t s_mem[kSeqArraysShare * kSeqsInLds];
    Arrays a = arrays_of(p.ws, p.b.n_seqs);
    const int n = p.b.n_seqs;
    if (n <= kSeqsInLds) {                // chains of loads and stores are faster there
        Arrays in = a;
        in.lead = s_mem;
        in.common = in.lead + n;
        in.members = in.common + n;
        in.least = in.members + n;
        in.total = in.least + n;
        in.next = in.total + n;
        for (int i = threadIdx.x; i < n; i += kThreads) {
            in.lead[i] = a.lead[i];
            in.common[i] = a.common[i];
            in.members[i] = a.members[i];
            in.least[i] = a.least[i];
            in.total[i] = a.total[i];
        }
        __syncthreads();
        list_groups(p, in);
    } else {
        list_groups(p, a);
    }
}

}  // namespace

size_t share_ws_bytes(int n_seqs) { return up256(words_of(n_seqs) * 4); }

hipError_t launch_share(const ShareParams &p, hipStream_t s)
{
    const int n = p.b.n_seqs;
    const int64_t rounds = (int64_t)n * ((p.b.max_pages + 64 * kWide - 1) / (64 * kWide));
    if (n <= kSeqsInLds && rounds <= kOneLaunch) {
        hipLaunchKernelGGL(share_kernel, dim3(1), dim3(kThreads), 0, s, p);
    } else {
        hipLaunchKernelGGL(lead_kernel, dim3(1), dim3(kThreads), 0, s, p);
        hipLaunchKernelGGL(common_kernel, dim3((n + 3) / 4), dim3(256), 0, s, p);
        hipLaunchKernelGGL(place_kernel, dim3(1), dim3(kThreads), 0, s, p);
    }
    return hipGetLastError();
}

}  // namespace lora
