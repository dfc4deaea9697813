// How the work of an attention call is divided as far as the host decides it: which kernels run, how many workgroups they may
// need, and the workspace.  Host only, plain C++; the constants are the kernels' too.
#pragma once
#include <limits.h>
#include <stddef.h>
#include <stdint.h>

#include <algorithm>

namespace lora {

constexpr int kLongTile = 128;           // rows
constexpr int kUnitShift = 7;            // a unit is 128 tokens: a step of a workgroup's four waves
constexpr float kMostUnits = 1 << 29;    // on the line; units are doubled until there are no more
constexpr int kMostBlocks = 768;         // workgroups of short tiles: three on every CU
// Items of long tiles that fill the chip: one on every CU.  Two fit, but the second adds less than writing and joining the parts
// of more cuts costs (4 chunks of 64 rows over 2000 tokens, 32 / 8 heads: 34.5 us, with twice the items 37.4; 2 chunks of 512 rows
// over 1500: 56 and 74; 8 of 128 over 500: 27 and 50; one of 200 over 8000: 58.7 and 55.8)
constexpr int kLongTarget = 256;
constexpr int kMostItems = (1 << 24) - 1;    // workgroups of 256 threads: a launch has less than 2^32 threads
constexpr int kLongMinSplit = 512;       // tokens of a cut range at least
// rows x group up to which a sequence goes in short tiles, where all have as many and where they differ.  Long tiles are faster
// from 33 on where there are many sequences (32 of 12 rows and 4 heads each over 1500 tokens: 64.7 / 49.3 us in short / long tiles; 128 of 9
// to 16 rows over 300 - 4000: 286 - 324 / 179 - 196), and so for one new row of 34 to 64 heads that share K and V (64 sequences
// over 100 - 8000 tokens 36 - 41 / 25 - 29 us, 256 of them 94 - 108 / 74 - 87, three over 80000 55 / 41; but 8 of them 14 - 21 / 22 - 23, one 9 - 13 /
// 10 - 21).  A batch of both takes two kernels, one after the other (48 uneven sequences of up to 13 rows, 5 x 4 heads of
// 80: 38.2 us in short tiles, 49.8 in both).
constexpr int kShortEqual = 32, kShortLimit = 64;
constexpr int kInlineSeqs = 256;         // sequences up to which every workgroup makes the plan for itself, in LDS: one launch less
// 32-bit words of the plan in memory: of its head, and of each sequence
constexpr int kPlanHead = 8, kPlanArrays = 7;

inline size_t up256(size_t n) { return (n + 255) & ~(size_t)255; }

// Which kernels a batch takes, and upper bounds of their work, from what the host knows.
struct Kinds {
    bool has_short, has_long;
    int limit;                            // rows x group of a sequence that goes in short tiles
    int shift;                            // rows of a short tile, as a power of two
    int blocks;                           // workgroups that share the short tiles
    int64_t long_items;                   // of long tiles, at most
};

inline Kinds kinds_of(int n_seqs, int n_rows, int max_rows, int heads, int kv_heads, int dim)
{
    const int64_t group = heads / kv_heads;
    const int64_t most = max_rows > 0 ? std::min(max_rows, n_rows) : n_rows;
    Kinds k;
    // As many rows in every sequence: all go in long tiles or all in short ones.  Where that would take more workgroups than a launch may
    // have, and wherever rows differ, a sequence goes in long tiles only with more than kShortLimit rows x group.
    bool equal = max_rows > 0 && (int64_t)max_rows * n_seqs == n_rows;
    for (;; equal = false) {
        k.has_long = most * group > (equal ? kShortEqual : kShortLimit);
        k.has_short = !k.has_long || !equal;
        // a sequence with more rows than the host thought still has to go somewhere
        k.limit = !k.has_long ? INT_MAX : !k.has_short ? 0 : kShortLimit;
        // tiles of a head: one for every sequence with that many rows, and what its rows fill; cuts add less than the target
        const int64_t seqs = std::min<int64_t>(std::min(n_seqs, n_rows), n_rows * group / ((int64_t)k.limit + 1));
        k.long_items = kLongTarget + kv_heads * (seqs + n_rows * group / kLongTile);
        if (!equal || !k.has_long || k.long_items <= kMostItems) break;
    }
    // Beside long chunks the others are taken for decoding users, in tiles of 16 rows: 64 of them with one or two rows of 4 heads 274
    // and 287 us for the batch, in tiles of 32 297 and 307; with 5 rows 340 and 314, 12 rows 436 and 415, 16 rows 468 and 385; 8 of any 0 to 3 us apart.
    k.shift = !k.has_long && most * group > 16 && dim <= 128 ? 5 : 4;
    k.blocks = dim <= 128 && k.shift == 4 ? kMostBlocks : kMostBlocks / 3 * 2;
    return k;
}

struct AttnWs {
    size_t plan, short_ml, short_o, long_ml, long_o, bytes;
};

inline AttnWs attn_ws_of(int n_seqs, const Kinds &k, int dim)
{
    const size_t rows_s = k.has_short ? 2 * (size_t)k.blocks << k.shift : 0, rows_l = k.has_long ? 2 * (size_t)kLongTarget * kLongTile : 0;
    AttnWs w;
    w.plan = 0;
    w.short_ml = up256((kPlanHead + kPlanArrays * (size_t)n_seqs) * 4);
    w.short_o = w.short_ml + up256(rows_s * 8);
    w.long_ml = w.short_o + up256(rows_s * dim * 4);
    w.long_o = w.long_ml + up256(rows_l * 8);
    w.bytes = w.long_o + up256(rows_l * dim * 4);
    return w;
}

}  // namespace lora
