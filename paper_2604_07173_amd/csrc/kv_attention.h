// What the two attention kernels share: work items, and the plan that cuts long ranges.
//
// A tile is R rows of one sequence and one key/value head: row r is query head r % group of new token r / group,
// so the heads that share K and V share their loads.  Sequences with few rows go in tiles of kShortTile
// (kv_attention.hip), the others in tiles of kLongRows (kv_attention_long.hip).  A work item is a tile and a
// range of its visible tokens; the plan cuts long ranges into items that run in parallel, and join_kernel
// joins their results.
#pragma once
#include "kv_device.h"

namespace lora {

constexpr int kShortTile = 16, kLongTile = 128;   // rows
constexpr int kShortTarget = 2048, kLongTarget = 512;   // work items that fill the chip: longer ranges are cut into about as many
constexpr int kShortMinSplit = 256, kLongMinSplit = 512;   // tokens of a cut range at least
constexpr int kShortLimit = 64;          // rows x group up to which a sequence goes in short tiles
constexpr float kLn2 = 0.6931471805599453f;

constexpr int kInlineSeqs = 256;         // sequences up to which every workgroup makes the plan for itself, in LDS: one launch less

// The plan: a head of kPlanHead words, then kPlanArrays arrays over the sequences: work items and partial results before
// each sequence, of short and of long tiles, and rows x heads to join.
enum { kChunkShort, kChunkLong, kItemsShort, kItemsLong, kJoinUnits, kPlanHead = 8 };
enum { kBaseShort, kSlotShort, kBaseLong, kSlotLong, kBaseJoin, kPlanArrays };
constexpr int kInlineWords = kPlanHead + kPlanArrays * kInlineSeqs;

struct Seq {
    int rows, len, pos0;                 // new rows, length, position of the first new row
};

__device__ inline Seq seq_of(const KvRows &b, int s)
{
    Seq q;
    const int first = min(max(0, b.row_start[s]), b.n_rows);
    q.rows = max(0, min(b.row_start[s + 1], b.n_rows) - first);
    q.len = min(max(0, b.seq_len[s]), b.tokens_max);
    q.pos0 = q.len - q.rows;
    return q;
}

// Tiles of R rows that the sequence has (none if it goes in the other kind).
template <int R>
__device__ inline int tiles_of(const AttnParams &p, const Seq &q)
{
    const int n = q.rows * p.group;
    if ((n <= p.short_limit) != (R == kShortTile)) return 0;
    return (n + R - 1) / R;
}

// Most tokens that a tile of the sequence sees.
template <int R>
__device__ inline int reach_of(const AttnParams &p, const Seq &q)
{
    if (!p.window) return q.len;
    const int64_t most = (int64_t)p.window - 1 + min(q.rows, R / p.group + 2);
    return (int)min((int64_t)q.len, most);
}

__device__ inline int splits_of(int reach, int chunk) { return reach <= chunk ? 1 : (reach + chunk - 1) / chunk; }

// A tile's tokens [lo, hi), into how many items they are cut, and the tokens of each.
struct Range {
    int lo, hi, splits, each;
};

template <int R>
__device__ inline Range range_of(const AttnParams &p, const Seq &q, int tile, int chunk)
{
    const int i0 = tile * R / p.group, i1 = min(q.rows - 1, (tile * R + R - 1) / p.group);
    Range r;
    r.hi = p.causal ? max(0, min(q.len, q.pos0 + i1 + 1)) : q.len;
    r.lo = p.window ? max(0, q.pos0 + i0 - p.window + 1) : 0;
    if (r.lo >= r.hi) r.lo = r.hi = 0;
    r.splits = splits_of(r.hi - r.lo, chunk);
    // evenly, in multiples of 64, as the chunk is one: no cut is empty, as splits - 1 chunks are not enough
    r.each = r.splits == 1 ? r.hi - r.lo : ((r.hi - r.lo + r.splits - 1) / r.splits + 63) >> 6 << 6;
    return r;
}

// Makes the plan with a workgroup of THREADS, into LDS or the workspace: cuts the ranges so that all work items of a kind
// take about as long.  Rows that are no partition of the batch's give no work at all.
template <int THREADS>
__device__ inline void make_plan(const AttnParams &p, int32_t *plan, bool report)
{
    constexpr int WAVES = THREADS / 64;
    __shared__ int64_t s_work[2][WAVES];
    __shared__ int s_sum[kPlanArrays][WAVES];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int n = p.b.n_seqs;
    int64_t work[2] = {0, 0};
    unsigned bad = 0;
    for (int s = tid; s < n; s += THREADS) {
        const Seq q = seq_of(p.b, s);
        if (p.b.seq_len[s] != q.len) bad |= 1;
        const int first = p.b.row_start[s], end = p.b.row_start[s + 1];
        if (first < 0 || end < first || end > p.b.n_rows || (s == 0 && first != 0) || (s == n - 1 && end != p.b.n_rows)) bad |= 2;
        work[0] += (int64_t)tiles_of<kShortTile>(p, q) * reach_of<kShortTile>(p, q);
        work[1] += (int64_t)tiles_of<kLongTile>(p, q) * reach_of<kLongTile>(p, q);
    }
    if (bad && report) atomicOr(p.b.status, LORA_STATUS_BAD_LENGTH);
#pragma unroll
    for (int d = 32; d; d >>= 1) {
        work[0] += __shfl_xor(work[0], d);
        work[1] += __shfl_xor(work[1], d);
    }
    if (lane == 0) s_work[0][wave] = work[0], s_work[1][wave] = work[1];
    const bool no_rows = __syncthreads_or(bad & 2);
    int chunk[2];
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        int64_t all = 0;
        for (int w = 0; w < WAVES; ++w) all += s_work[k][w];
        const int64_t target = k ? kLongTarget : kShortTarget, least = k ? kLongMinSplit : kShortMinSplit;
        const int64_t each = (all * p.c.n_heads + target - 1) / target;
        chunk[k] = (int)min(((max(each, least) + 127) >> 7) << 7, (int64_t)1 << 30);
    }
    int base[kPlanArrays] = {};
    for (int s0 = 0; s0 < n; s0 += THREADS) {
        const int s = s0 + tid;
        int own[kPlanArrays] = {}, v[kPlanArrays];
        if (s < n && !no_rows) {
            const Seq q = seq_of(p.b, s);
            const int cut_s = splits_of(reach_of<kShortTile>(p, q), chunk[0]), cut_l = splits_of(reach_of<kLongTile>(p, q), chunk[1]);
            const int tiles_s = tiles_of<kShortTile>(p, q), tiles_l = tiles_of<kLongTile>(p, q);
            own[kBaseShort] = tiles_s * cut_s * p.c.n_heads;
            own[kSlotShort] = cut_s > 1 ? own[kBaseShort] : 0;
            own[kBaseLong] = tiles_l * cut_l * p.c.n_heads;
            own[kSlotLong] = cut_l > 1 ? own[kBaseLong] : 0;
            own[kBaseJoin] = (tiles_s ? cut_s : cut_l) > 1 ? q.rows * p.heads : 0;
        }
        __syncthreads();
#pragma unroll
        for (int k = 0; k < kPlanArrays; ++k) v[k] = own[k];
#pragma unroll
        for (int d = 1; d < 64; d <<= 1)
#pragma unroll
            for (int k = 0; k < kPlanArrays; ++k) {
                const int o = __shfl_up(v[k], d);
                if (lane >= d) v[k] += o;
            }
        if (lane == 63)
#pragma unroll
            for (int k = 0; k < kPlanArrays; ++k) s_sum[k][wave] = v[k];
        __syncthreads();
#pragma unroll
        for (int k = 0; k < kPlanArrays; ++k) {
            int total = 0;
            for (int w = 0; w < WAVES; ++w) {
                if (w < wave) v[k] += s_sum[k][w];
                total += s_sum[k][w];
            }
            if (s < n) plan[kPlanHead + k * n + s] = base[k] + v[k] - own[k];
            base[k] += total;
        }
    }
    if (tid == 0) {
        plan[kChunkShort] = chunk[0];
        plan[kChunkLong] = chunk[1];
        plan[kItemsShort] = base[kBaseShort];
        plan[kItemsLong] = base[kBaseLong];
        plan[kJoinUnits] = base[kBaseJoin];
    }
    __syncthreads();
}

// The plan of a workgroup of 256: made in s_plan, or what a launch before has left in the workspace.
__device__ inline const int32_t *plan_of(const AttnParams &p, int32_t *s_plan)
{
    if (p.b.n_seqs > kInlineSeqs) return p.plan;
    make_plan<256>(p, s_plan, blockIdx.x == 0);
    return s_plan;
}

struct Item {
    int s, head, tile, cut, cuts, slot;
};

// Work item n: the cuts of a tile lie n_heads apart, tiles behind each other.
template <int R>
__device__ inline Item item_of(const AttnParams &p, const int32_t *plan, int n, Seq &q)
{
    const int32_t *base = plan + kPlanHead + (R == kShortTile ? kBaseShort : kBaseLong) * p.b.n_seqs;
    Item it;
    it.s = wave_find(base, p.b.n_seqs, n);
    q = seq_of(p.b, it.s);
    const int left = n - base[it.s];
    it.slot = base[p.b.n_seqs + it.s] + left;
    const int pair = left / p.c.n_heads;
    it.head = left - pair * p.c.n_heads;
    it.cuts = splits_of(reach_of<R>(p, q), plan[R == kShortTile ? kChunkShort : kChunkLong]);
    it.tile = pair / it.cuts;
    it.cut = pair - it.tile * it.cuts;
    return it;
}

// Any of eight bf16 that is no finite number.
__device__ inline bool not_finite(u32x4 v)
{
    bool r = false;
#pragma unroll
    for (int i = 0; i < 4; ++i) r |= (v[i] & 0x7F800000u) == 0x7F800000u || (v[i] & 0x7F80u) == 0x7F80u;
    return r;
}

// Eight bf16 with zeros for those that are no finite numbers, and the other part of one.
__device__ inline bf16x8 finite_part(bf16x8 v8)
{
    u32x4 v = __builtin_bit_cast(u32x4, v8);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if ((v[i] & 0x7F800000u) == 0x7F800000u) v[i] &= 0x0000FFFFu;
        if ((v[i] & 0x7F80u) == 0x7F80u) v[i] &= 0xFFFF0000u;
    }
    return as_bf16x8(v);
}

__device__ inline float odd_part(uint16_t v)
{
    return (v & 0x7F80u) == 0x7F80u ? __uint_as_float((unsigned)v << 16) : 0.f;
}

// K and V lie in LDS as rows of DP elements; the 16-byte pieces of a row change places by its number, so that
// eight rows' pieces of one column, and four rows' pairs of pieces, lie in different banks.
template <int DP>
__device__ inline int swizzled(int row, int piece)
{
    return DP == 64 ? piece ^ ((row >> 1 & 3) << 1) : piece ^ ((row & 7) << 1);
}

// Four elements of each of four rows, transposed within 16 lanes: lane 4 r + c gives the address of elements 4 c .. 4 c + 3
// of row r, and lane n receives column n.
__device__ inline u32x2 read_transposed(const uint16_t *at)
{
    typedef __attribute__((ext_vector_type(4))) short s16x4;
    typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
    return __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)at));
}

hipError_t launch_attend_long(const AttnParams &p, int max_items, hipStream_t s);

}  // namespace lora
