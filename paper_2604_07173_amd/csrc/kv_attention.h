// What the two attention kernels share: tiles, and the plan that divides the work.
//
// A tile is a number of rows of one sequence and one key/value head: row r is query head r % group of new token
// r / group, so the heads that share K and V share their loads.  Sequences with few rows go in tiles of 16 or 32 rows
// (kShort, kv_attention.hip), the others in tiles of kLongTile (kLong, kv_attention_long.hip).
//
// Short tiles are bound by the reading of K and V.  All their tokens, in units of 128 per tile, form one line, and every
// workgroup takes an equal stretch of it, whatever the lengths are: several tiles, or a part of a long one.  Tiles that
// lie across the end of a stretch leave partial results, two at most per workgroup, which join_kernel joins.
//
// Long tiles are work items of their own; where there are few, their tokens are cut evenly into several items.
#pragma once
#include "kv_device.h"
#include "kv_work.h"

namespace lora {

constexpr float kLn2 = 0.6931471805599453f;

enum Kind { kShort, kLong };

// The plan: a head of kPlanHead words, then kPlanArrays arrays over the sequences: units of short tiles before each
// sequence, work items and partial results of long tiles, and rows x heads of long tiles to join; then the sequences
// themselves.
enum { kUnits, kShare, kUnitTokens, kChunk, kItems, kJoinUnits, kHeadWords };
enum { kBaseUnit, kBaseItem, kBaseSlot, kBaseJoin, kPlanSums, kSeqRow0 = kPlanSums, kSeqRows, kSeqLen, kSeqArrays };
static_assert(kHeadWords <= kPlanHead && kSeqArrays == kPlanArrays, "as many words as the host makes room for");
constexpr int kInlineWords = kPlanHead + kPlanArrays * kInlineSeqs;

struct Seq {
    int row0, rows, len, pos0;           // first new row and their number, length, position of the first new row
};

__device__ inline Seq seq_of(const KvRows &b, int s)
{
    Seq q;
    q.row0 = min(max(0, b.row_start[s]), b.n_rows);
    q.rows = max(0, min(b.row_start[s + 1], b.n_rows) - q.row0);
    q.len = min(max(0, b.seq_len[s]), b.tokens_max);
    q.pos0 = q.len - q.rows;
    return q;
}

template <Kind K>
__device__ inline int tile_rows(const AttnParams &p) { return K == kShort ? 1 << p.short_shift : kLongTile; }

// Tiles that the sequence has of this kind.
template <Kind K>
__device__ inline int tiles_of(const AttnParams &p, const Seq &q)
{
    const int n = q.rows * p.group;
    if ((n <= p.short_limit) != (K == kShort)) return 0;
    return K == kShort ? (n + (1 << p.short_shift) - 1) >> p.short_shift : (n + kLongTile - 1) / kLongTile;
}

// Most tokens that a tile of the sequence sees.
template <Kind K>
__device__ inline int reach_of(const AttnParams &p, const Seq &q)
{
    if (!p.window) return q.len;
    const int most = p.window - 1 + min(q.rows, tile_rows<K>(p) / p.group_div + 2);
    return min(q.len, most);
}

__device__ inline int splits_of(int reach, int chunk) { return reach <= chunk ? 1 : (reach + chunk - 1) / chunk; }

__device__ inline int units_of(int reach, int shift) { return max(1, (reach + (1 << shift) - 1) >> shift); }

// Tokens of a unit, as a power of two.  `units`: of 128 tokens, all of the line.
__device__ inline int unit_shift_of(float units)
{
    int shift = kUnitShift;
    for (; units > kMostUnits && shift < 30; units *= 0.5f) ++shift;
    return shift;
}

// A tile's tokens [lo, hi).
struct Range {
    int lo, hi;
};

template <Kind K>
__device__ inline Range range_of(const AttnParams &p, const Seq &q, int tile)
{
    const int R = tile_rows<K>(p);
    const int i0 = tile * R / p.group_div, i1 = min(q.rows - 1, (tile * R + R - 1) / p.group_div);
    Range r;
    r.hi = p.causal ? max(0, min(q.len, q.pos0 + i1 + 1)) : q.len;
    r.lo = p.window ? max(0, q.pos0 + i0 - p.window + 1) : 0;
    if (r.lo >= r.hi) r.lo = r.hi = 0;
    return r;
}

// Tokens of an item of a cut tile.  `work`: tokens that all long tiles of a key/value head see.  A little more than the
// even share, so that the number of cut items stays below twice the target however it was rounded; a tile is
// only cut where that fills the chip better.
__device__ inline int chunk_of(const AttnParams &p, float work)
{
    const float each = work * (float)p.c.n_heads * (1.25f / kLongTarget);
    return each < (float)kLongMinSplit ? kLongMinSplit : each > 1e9f ? 1 << 30 : ((int)each + 128) >> 7 << 7;
}

// Tokens of each cut, evenly, in multiples of 64, as the chunk is one: no cut is empty, as splits - 1 chunks are not enough.
__device__ inline int cut_of(const Range &r, int splits)
{
    return splits == 1 ? r.hi - r.lo : ((r.hi - r.lo + splits - 1) / splits + 63) >> 6 << 6;
}

// What a sequence adds to the plan's arrays.
__device__ inline void plan_entry(const AttnParams &p, const Seq &q, int shift, int chunk, int (&own)[kPlanSums])
{
    const int tiles = tiles_of<kLong>(p, q);
    const int cuts = splits_of(reach_of<kLong>(p, q), chunk);
    own[kBaseUnit] = tiles_of<kShort>(p, q) * p.c.n_heads * units_of(reach_of<kShort>(p, q), shift);
    own[kBaseItem] = tiles * cuts * p.c.n_heads;
    own[kBaseSlot] = cuts > 1 ? own[kBaseItem] : 0;
    own[kBaseJoin] = cuts > 1 && tiles ? q.rows * p.heads : 0;
}

__device__ inline void plan_head(const AttnParams &p, int32_t *plan, int shift, int chunk, const int (&sum)[kPlanSums])
{
    plan[kUnits] = sum[kBaseUnit];
    plan[kShare] = max(1, (sum[kBaseUnit] + p.short_blocks - 1) / p.short_blocks);
    plan[kUnitTokens] = shift;
    plan[kChunk] = chunk;
    plan[kItems] = sum[kBaseItem];
    plan[kJoinUnits] = sum[kBaseJoin];
}

__device__ inline void store_seq(int32_t *plan, int64_t n_seqs, int s, const Seq &q)
{
    plan[kPlanHead + kSeqRow0 * n_seqs + s] = q.row0;
    plan[kPlanHead + kSeqRows * n_seqs + s] = q.rows;
    plan[kPlanHead + kSeqLen * n_seqs + s] = q.len;
}

__device__ inline Seq planned_seq(const int32_t *plan, int64_t n_seqs, int s)
{
    Seq q;
    q.row0 = uniform(plan[kPlanHead + kSeqRow0 * n_seqs + s]);
    q.rows = uniform(plan[kPlanHead + kSeqRows * n_seqs + s]);
    q.len = uniform(plan[kPlanHead + kSeqLen * n_seqs + s]);
    q.pos0 = q.len - q.rows;
    return q;
}

// Rows of sequence s that are no part of a partition of the batch's (2), a length that the table cannot hold (1).
__device__ inline unsigned faults_of(const KvRows &b, int s)
{
    const int first = b.row_start[s], end = b.row_start[s + 1], len = b.seq_len[s];
    unsigned bad = len < 0 || len > b.tokens_max;
    if (first < 0 || end < first || end > b.n_rows || (s == 0 && first != 0) || (s == b.n_seqs - 1 && end != b.n_rows)) bad |= 2;
    return bad;
}

// The plan of up to kInlineSeqs sequences, by one wave: lane l takes the sequences l * each .. of the batch.
__device__ inline void make_plan(const AttnParams &p, int32_t *plan)
{
    constexpr int MOST = kInlineSeqs / 64;
    const int lane = threadIdx.x & 63, n = p.b.n_seqs, each = (n + 63) >> 6;
    Seq q[MOST];
    unsigned bad = 0;
    float work = 0.f;
#pragma unroll
    for (int k = 0; k < MOST; ++k) {
        const int s = lane * each + k;
        q[k] = Seq{0, 0, 0, 0};
        if (k < each && s < n) {
            q[k] = seq_of(p.b, s);
            bad |= faults_of(p.b, s);
        }
    }
    float units = 0.f;
#pragma unroll
    for (int k = 0; k < MOST; ++k) units += (float)(tiles_of<kShort>(p, q[k]) * p.c.n_heads) * (float)units_of(reach_of<kShort>(p, q[k]), kUnitShift);
    const int shift = unit_shift_of(last_lane(wave_scan(units)));
    int chunk = 1 << 30;
    if (p.long_o) {
#pragma unroll
        for (int k = 0; k < MOST; ++k) work += (float)tiles_of<kLong>(p, q[k]) * (float)reach_of<kLong>(p, q[k]);
        chunk = chunk_of(p, last_lane(wave_scan(work)));
    }
    int own[MOST][kPlanSums] = {}, sum[kPlanSums] = {};
    if (!__any(bad & 2)) {                // rows that are no partition: no work at all
#pragma unroll
        for (int k = 0; k < MOST; ++k) {
            if (k >= each) break;
            plan_entry(p, q[k], shift, chunk, own[k]);
#pragma unroll
            for (int a = 0; a < kPlanSums; ++a) sum[a] += own[k][a];
        }
    }
#pragma unroll
    for (int a = 0; a < kPlanSums; ++a) {
        const int upto = wave_scan(sum[a]);
        int before = upto - sum[a];
        sum[a] = upto;                    // lane 63's is the total
#pragma unroll
        for (int k = 0; k < MOST; ++k) {
            const int s = lane * each + k;
            if (k < each && s < n) plan[kPlanHead + a * n + s] = before;
            before += own[k][a];
        }
    }
#pragma unroll
    for (int k = 0; k < MOST; ++k)
        if (k < each && lane * each + k < n) store_seq(plan, n, lane * each + k, q[k]);
    if (lane == 63) plan_head(p, plan, shift, chunk, sum);
    if (bad && blockIdx.x == 0) atomicOr(p.b.status, LORA_STATUS_BAD_LENGTH);
}

// The plan: made in s_plan by the workgroup's first wave, or what plan_kernel has left in the workspace.  The first workgroup
// leaves its own there for the launch after.
__device__ inline const int32_t *plan_of(const AttnParams &p, int32_t *s_plan)
{
    if (p.b.n_seqs > kInlineSeqs) return p.plan;
    if (threadIdx.x < 64) make_plan(p, s_plan);
    __syncthreads();
    if (blockIdx.x == 0)
        for (int i = threadIdx.x; i < kPlanHead + kPlanArrays * p.b.n_seqs; i += blockDim.x) p.plan[i] = s_plan[i];
    return s_plan;
}

// The sequence that entry n of one of the plan's arrays belongs to.
__device__ inline int seq_at(const AttnParams &p, const int32_t *base, int n)
{
    return __builtin_amdgcn_readfirstlane(p.b.n_seqs == 1 ? 0 : wave_find(base, p.b.n_seqs, n));
}

// A tile on the line of units.
struct Place {
    int s, head, tile, start, units;     // start: the tile's first unit on the line
};

__device__ inline Place place_of(const AttnParams &p, const int32_t *plan, int unit, Seq &q)
{
    const int32_t *base = plan + kPlanHead + kBaseUnit * p.b.n_seqs;
    Place x;
    x.s = seq_at(p, base, unit);
    q = planned_seq(plan, p.b.n_seqs, x.s);
    x.units = units_of(reach_of<kShort>(p, q), uniform(plan[kUnitTokens]));
    const int before = uniform(base[x.s]);
    const int pair = x.units == 1 ? unit - before : (unit - before) / x.units;
    x.start = before + pair * x.units;
    x.tile = pair / p.kv_div;
    x.head = pair - x.tile * p.c.n_heads;
    return x;
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
