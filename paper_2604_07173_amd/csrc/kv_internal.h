// Internal declarations of the paged cache, its append, attention and page calls (host side; kernels
// live in kv_append.hip, kv_attention.hip and kv_pages.hip).
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "../../include/lora_attn.h"
#include "lora_layout.h"

namespace lora {

int note_hip_error(hipError_t e);   // keeps the text for lora_last_hip_error; returns LORA_ERR_HIP

// One layer of a cache.
struct KvView {
    uint16_t *k, *v;
    int64_t page_stride, head_stride, token_stride;   // elements
    int n_pages, page_shift, n_heads, dim;
};

// The sequences of a batch.  tokens_max: what a table row can hold.
struct KvRows {
    const int32_t *row_start, *seq_len, *table, *position;
    uint32_t *status;
    int n_seqs, n_rows, max_pages, tokens_max;
};

// Groups of sequences that hold the same first pages, as lora_kv_shared says.  most: room for groups; most_rows: for their rows.
struct KvGroups {
    const int32_t *groups, *rows, *own, *place, *counts;
    int most, most_rows;
};

struct AppendParams {
    KvView c;
    KvRows b;
    const void *q, *k, *v;
    int64_t ldq, ldk, ldv, ldqo;
    uint16_t *q_out;
    const double *freq;
    float amplitude;
    int rot, pairing, heads;      // heads: of q, 0 = no q
    int kv_heads;                 // of k and v, 0 = no append
    int f32;
};

struct AttnParams {
    KvView c;
    KvRows b;
    const uint16_t *q;
    uint16_t *out;
    float *lse;
    int64_t ldq, ldo;
    float scale_log2;             // scale / ln 2
    int heads, group, causal, window;
    FastDiv group_div, kv_div, heads_div;
    int short_limit;              // rows x group of a sequence up to which it goes in short tiles
    int short_shift;              // rows of a short tile, as a power of two
    int short_blocks, join_blocks;   // workgroups that share the short tiles, and that join their parts
    int32_t *plan;                // device: see kv_attention.h
    float *part_o, *part_ml;      // partial results of short tiles whose range is cut: sums, and maximum and sum of weights
    float *long_o, *long_ml;
    // lora_kv_attention_shared only
    KvGroups g;
    int group_limit;              // as short_limit, of a group's rows
    float *whole_o, *whole_ml;    // of groups' rows and heads: over the shared tokens, then over their own
    int4 *found;                  // of the same: where their parts are (kv_attention.h)
    int parts_short, parts_long;  // partial results that there is room for
    // (behind the others, whose places decide how the attention kernels' registers are loaded: in front of `plan` it cost one 5 %)
    int join_long;                // workgroups that join long tiles' parts
};

struct ShareParams {
    KvRows b;
    int32_t *groups, *rows, *own, *place, *counts;
    int32_t *ws;
    int page_shift, min_pages, max_rows, most, most_rows;
};

struct PlanParams {
    const int32_t *from_table, *from_len, *from_ref;
    int32_t *to_table, *to_len, *to_ref;
    const int32_t *src, *new_len;
    int32_t *pairs, *counts;
    uint32_t *status;
    int32_t *ws;
    int n_pages, n_seqs, max_pages, page_shift;
};

struct CopyParams {
    uint16_t *k, *v;
    const int32_t *pairs, *counts;
    int64_t layer_stride, page_stride, inner_stride, outer_stride;   // elements
    int run, inner, outer;        // a page is outer x inner runs of `run` elements
    FastDiv run_vecs, inner_div;
    int n_layers, n_pages, max_moves;
};

hipError_t launch_append(const AppendParams &p, hipStream_t s);
size_t attention_ws_bytes(int n_seqs, int n_rows, int max_rows, int heads, int kv_heads, int dim);
hipError_t launch_attention(AttnParams &p, int max_rows, void *ws, hipStream_t s);
size_t attention_shared_ws_bytes(int n_seqs, int n_rows, int max_rows, int group_rows, int max_group_rows, int heads, int kv_heads, int dim);
hipError_t launch_attention_shared(AttnParams &p, int max_rows, int max_group_rows, void *ws, hipStream_t s);
size_t share_ws_bytes(int n_seqs);
hipError_t launch_share(const ShareParams &p, hipStream_t s);
size_t plan_ws_bytes(int n_pages, int n_seqs);
hipError_t launch_plan(const PlanParams &p, hipStream_t s);
hipError_t launch_compact(const PlanParams &p, hipStream_t s);
hipError_t launch_copy_pages(const CopyParams &p, hipStream_t s);

}  // namespace lora
