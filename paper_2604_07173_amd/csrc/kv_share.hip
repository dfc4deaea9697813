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
// Rounds of comparing that the waves of one workgroup take on, at most: sequences x their rounds.
constexpr int kOneLaunch = 8 * kWaves;

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

// Leading table entries of sequence s that agree with its leader's, by a wave.
__device__ inline void compare(const ShareParams &p, const Arrays &a, int s)
{
    const int lane = threadIdx.x & 63, lead = uniform(a.lead[s]);
    int common = 0;
    if (lead >= 0) {
        const Seq q = seq_of(p, s);
        common = min(q.whole, seq_of(p, lead).whole);
        const int32_t *mine = p.b.table + (int64_t)s * p.b.max_pages, *its = p.b.table + (int64_t)lead * p.b.max_pages;
        for (int at = 0; at < common && s != lead; at += 64 * kWide) {
            int x[kWide], y[kWide];
#pragma unroll
            for (int k = 0; k < kWide; ++k) {
                const int i = min(at + k * 64 + lane, common - 1);
                x[k] = mine[i];
                y[k] = its[i];
            }
            int differ = INT_MAX;
#pragma unroll
            for (int k = kWide - 1; k >= 0; --k) {
                const u64 mask = __ballot(x[k] != y[k]);
                if (mask) differ = at + k * 64 + __ffsll(mask) - 1;
            }
            if (differ < common) common = differ;      // which ends the loop
        }
        if (lane == 0 && common >= p.min_pages) {
            atomicAdd(&a.members[lead], 1);
            atomicMin(&a.least[lead], common);
            atomicAdd(&a.total[lead], q.rows);
        }
    }
    if (lane == 0) a.common[s] = common;
}

__device__ inline void list_groups(const ShareParams &p, const Arrays &a)
{
    const int n = p.b.n_seqs, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    int groups = 0, rows = 0, in = 0;
    int64_t spared = 0;
    for (int s0 = 0; s0 < n; s0 += kThreads) {
        const int s = s0 + tid;
        int members = 0, total = 0, least = 0;
        if (s < n && a.lead[s] == s) {
            members = fresh(&a.members[s]);
            total = fresh(&a.total[s]);
            least = fresh(&a.least[s]);
        }
        const bool head = members >= 2;
        int sum_groups, sum_rows, sum_in;
        int64_t sum_spared;
        const int number = groups + block_scan<kWaves>(head ? 1 : 0, sum_groups) - 1;
        const int first = rows + block_scan<kWaves>(head ? total : 0, sum_rows) - total;
        block_scan<kWaves>(head ? members : 0, sum_in);
        block_scan<kWaves>(head ? (int64_t)(members - 1) * ((int64_t)least << p.page_shift) : (int64_t)0, sum_spared);
        if (head) {
            int32_t *g = p.groups + 4 * (int64_t)number;
            g[0] = s;
            g[1] = least << p.page_shift;
            g[2] = first;
            g[3] = total;
            a.next[s] = first;
        }
        groups += sum_groups;
        rows += sum_rows;
        in += sum_in;
        spared += sum_spared;
    }
    if (tid == 0) {
        p.counts[0] = groups;
        p.counts[1] = rows;
        p.counts[2] = in;
        p.counts[3] = (int32_t)min(spared, (int64_t)INT_MAX);
    }
    for (int64_t i = 4 * (int64_t)groups + tid; i < 4 * (int64_t)p.most; i += kThreads) p.groups[i] = i & 3 ? 0 : -1;
    for (int i = rows + tid; i < p.most_rows; i += kThreads) p.rows[i] = -1;
    __syncthreads();
    for (int s0 = 0; s0 < n; s0 += kThreads) {
        const int s = s0 + tid;
        int lead = s < n ? a.lead[s] : -1;
        if (lead >= 0 && (a.common[s] < p.min_pages || fresh(&a.members[lead]) < 2)) lead = -1;
        const Seq q = lead >= 0 ? seq_of(p, s) : Seq{};
        // rows of this wave's members of the same group: those before this one, and all; whether this is the last of them
        int before = 0, all = 0, last = lane;
        for (int j = 0; j < 64; ++j) {
            const int other = __builtin_amdgcn_readlane(lead, j), its = __builtin_amdgcn_readlane(q.rows, j);
            if (other != lead || lead < 0) continue;
            if (j < lane) before += its;
            all += its;
            last = j;
        }
        // one wave after another takes its part of every group's rows
        int at = -1;
        const int waves = min(kWaves, (n - s0 + 63) >> 6);
        for (int w = 0; w < waves; ++w) {
            if (w == wave && lead >= 0) {
                const int base = a.next[lead];
                at = base + before;
                if (last == lane) a.next[lead] = base + all;
            }
            __syncthreads();
        }
        if (s < n) {
            p.own[s] = lead < 0 ? 0 : fresh(&a.least[lead]) << p.page_shift;
            p.place[s] = at;
            for (int i = 0; i < q.rows; ++i) p.rows[at + i] = p.b.row_start[s] + i;
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
    for (int s = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6); s < p.b.n_seqs; s += kWaves) compare(p, a, s);
    __syncthreads();
    list_groups(p, a);
}

__global__ __launch_bounds__(kThreads) void lead_kernel(ShareParams p) { find_leaders(p, arrays_of(p.ws, p.b.n_seqs)); }

__global__ __launch_bounds__(256) void common_kernel(ShareParams p)
{
    const Arrays a = arrays_of(p.ws, p.b.n_seqs);
    const int s = __builtin_amdgcn_readfirstlane(blockIdx.x * 4 + (threadIdx.x >> 6));
    if (s < p.b.n_seqs) compare(p, a, s);
}

__global__ __launch_bounds__(kThreads) void place_kernel(ShareParams p) { list_groups(p, arrays_of(p.ws, p.b.n_seqs)); }

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
