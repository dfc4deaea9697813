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

// The device plan: a head of kPlanHead words, then four arrays over the sequences.
enum { kChunkShort, kChunkLong, kItemsShort, kItemsLong, kPlanHead = 16 };

struct Plan {
    const int32_t *head, *base, *slot;   // work items and partial results before each sequence
    int chunk, items;
};

template <int R>
__device__ inline Plan plan_of(const AttnParams &p)
{
    constexpr bool SHORT = R == kShortTile;
    Plan q;
    q.head = p.plan;
    q.base = p.plan + kPlanHead + (SHORT ? 0 : 2) * p.b.n_seqs;
    q.slot = q.base + p.b.n_seqs;
    q.chunk = p.plan[SHORT ? kChunkShort : kChunkLong];
    q.items = p.plan[SHORT ? kItemsShort : kItemsLong];
    return q;
}

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

struct Item {
    int s, head, tile, cut, cuts, slot;
};

// Work item n: the cuts of a tile lie n_heads apart, tiles behind each other.
template <int R>
__device__ inline Item item_of(const AttnParams &p, const Plan &plan, int n, Seq &q)
{
    Item it;
    it.s = wave_find(plan.base, p.b.n_seqs, n);
    q = seq_of(p.b, it.s);
    const int left = n - plan.base[it.s];
    it.slot = plan.slot[it.s] + left;
    const int pair = left / p.c.n_heads;
    it.head = left - pair * p.c.n_heads;
    it.cuts = splits_of(reach_of<R>(p, q), plan.chunk);
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
