/*
 * What stands between the q/k/v and the output projection of an attention layer: rotary positions
 * with the append to a paged cache, attention of new rows over that cache, and the bookkeeping of
 * its pages.  Together with lora_apply_group (q, k, v) and lora_apply (output) of lora.h it is the
 * attention block of an LLM instance whose adapters are served from a pool (Sec. 2.2, Sec. 5).
 *
 * The conventions of lora.h hold: status codes and no exceptions, device memory owned by the
 * caller, all work on `stream` and nothing that waits, host-detectable mistakes before any device
 * work.  Mistakes that only the device can see (a page outside the cache, a length beyond the
 * table) raise a bit in the status word of the call's structure, which the calls only ever add to
 * and the caller clears; nothing is read or written out of bounds then.
 */
#ifndef LORA_ATTN_H
#define LORA_ATTN_H

#include "lora.h"

#ifdef __cplusplus
extern "C" {
#endif

enum {
    LORA_KV_MAX_HEAD_DIM = 256,
    LORA_KV_MAX_PAGE = 1024,      /* tokens of a page */
    LORA_KV_MAX_PAGES = 0x7FFFFC00,      /* pages of a cache: chunks of 1024 are numbered in 32 bits */
    LORA_KV_MAX_GROUP = 64        /* query heads that share a key/value head */
};

/* further bits of a device status word */
enum {
    LORA_STATUS_BAD_PAGE = 4u,    /* a table entry in use is not a page of the cache */
    LORA_STATUS_BAD_LENGTH = 8u,  /* a length is negative or beyond the table, or row_start
                                     is no partition of the rows */
    LORA_STATUS_BAD_SEQ = 16u,    /* lora_kv_plan: src names no slot */
    LORA_STATUS_NO_PAGES = 32u    /* lora_kv_plan: fewer free pages than asked for */
};

/* ------------------------------------------------------------------------------------
 * The cache: K and V in bf16, cut into pages of page_size tokens of all key/value heads.  Element
 * (layer, page, head, token, d) of K is at k + layer * layer_stride + page * page_stride +
 * head * head_stride + token * token_stride + d, of V likewise; strides are in elements and
 * multiples of 8, and layers, pages, heads and tokens may lie in any order in which each begins beyond
 * what those with smaller strides span (LORA_ERR_BAD_SHAPE); of what there is one, any multiple of 8
 * will do.  The last element is less than 2^61 elements from the first (LORA_ERR_TOO_LARGE).  k and v
 * are 16-byte aligned device memory.  n_pages: 1 .. LORA_KV_MAX_PAGES.  page_size: a power of two,
 * 1 .. LORA_KV_MAX_PAGE.  head_dim: a multiple of 8, 8 .. LORA_KV_MAX_HEAD_DIM.  All layers share the
 * tables.
 * ------------------------------------------------------------------------------------ */
typedef struct lora_kv_cache {
    void *k, *v;
    int32_t n_layers, n_pages, n_heads, page_size, head_dim;
    int32_t reserved;
    int64_t layer_stride, page_stride, head_stride, token_stride;
} lora_kv_cache;

/*
 * The sequences of a batch and their new rows.  Rows row_start[s] .. row_start[s + 1] - 1 are
 * the new tokens of sequence s, the last of its seq_len[s] tokens (new ones included): row i of
 * its n stands at position seq_len[s] - n + i.  Token p of sequence s is in page
 * table[s * max_pages + p / page_size], at place p % page_size.  A sequence may have no rows.
 * row_start[0] = 0, row_start does not fall, row_start[n_seqs] = n_rows; if not, attention raises
 * LORA_STATUS_BAD_LENGTH and writes nothing, and lora_rope_append raises it for rows of no sequence and
 * leaves them out of the cache.
 */
typedef struct lora_kv_batch {
    int32_t n_seqs;             /* >= 1 */
    int32_t n_rows;             /* new rows of all sequences, at most LORA_MAX_ROWS_LONG */
    int32_t max_rows;           /* rows of the longest sequence as far as the host knows, 0 = unknown;
                                   decides which kernels run, and so how sums are
                                   rounded, but nothing else */
    int32_t max_pages;          /* entries of a table row */
    const int32_t *row_start;   /* device [n_seqs + 1] */
    const int32_t *seq_len;     /* device [n_seqs] */
    const int32_t *table;       /* device [n_seqs][max_pages] */
    const int32_t *position;    /* device [n_rows] or NULL: what lora_rope_append rotates by in place of
                                   the row's place in its sequence; may be negative */
    uint32_t *status;           /* device [1] */
} lora_kv_batch;

/* ------------------------------------------------------------------------------------
 * Rotary positions.
 *
 * The first rot_dim elements of a head are rot_dim / 2 pairs: LORA_ROPE_HALF pairs element i with
 * i + rot_dim / 2, LORA_ROPE_INTERLEAVED 2 i with 2 i + 1.  At position p pair i becomes
 *   (a, b) -> amplitude * (a cos t - b sin t, a sin t + b cos t),   t = p * freq[i];
 * elements from rot_dim on pass.  The same call with positions negated is the inverse (and the
 * gradient) up to the square of the amplitude.  The angle is formed in 64 bits and reduced to one
 * turn before it is rounded, so that it is as exact at position 10^6 as at 0.
 *
 * lora_rope_freqs (host): freq[i] = base^(-2 i / rot_dim), then by `scaling`
 *   LORA_ROPE_PLAIN    nothing more
 *   LORA_ROPE_LINEAR   divided by factor
 *   LORA_ROPE_BASE     base * factor^(rot_dim / (rot_dim - 2)) in place of base
 *   LORA_ROPE_PARTS    g * freq + (1 - g) * freq / factor, with g = 0 for pairs that turn less
 *                      than `low` times in original_len positions, 1 from `high` times on, and
 *                      linear in the number of turns between
 * ------------------------------------------------------------------------------------ */
enum { LORA_ROPE_HALF = 0, LORA_ROPE_INTERLEAVED = 1 };
enum { LORA_ROPE_PLAIN = 0, LORA_ROPE_LINEAR = 1, LORA_ROPE_BASE = 2, LORA_ROPE_PARTS = 3 };

typedef struct lora_rope_desc {
    int32_t rot_dim;      /* even, 2 .. LORA_KV_MAX_HEAD_DIM */
    int32_t scaling;
    double base;          /* > 1 */
    double factor;        /* >= 1 */
    double original_len;  /* LORA_ROPE_PARTS: > 0 */
    double low, high;     /* LORA_ROPE_PARTS: 0 <= low < high */
} lora_rope_desc;

int lora_rope_freqs(const lora_rope_desc *d, double *freq);   /* host [rot_dim / 2] */

typedef struct lora_rope {
    const double *freq;   /* device [rot_dim / 2], 8-byte aligned */
    int32_t rot_dim;      /* even, 2 .. head_dim of the cache */
    int32_t pairing;
    float amplitude;
    int32_t reserved;
} lora_rope;

/*
 * Rotates q [n_rows][n_heads * head_dim] into q_out (bf16) and k into the cache's pages of the
 * batch's rows, and puts v there as it is.  in_dtype: LORA_DTYPE_BF16 or LORA_DTYPE_F32 (the
 * outputs of lora_expand in 32 bits), for q, k and v; everything is rounded to bf16 once, to
 * nearest even.  ldq, ldk, ldv, ldqo: row strides in elements, multiples of 8, so the inputs
 * may be column ranges of one buffer.  q NULL: only the append (q_out, n_heads ignored).  k and
 * v both NULL: only q.  rope NULL: nothing is rotated.  q_out may be q itself (bf16, ldqo ==
 * ldq); other overlaps of inputs and outputs are not allowed.  Two sequences that write to one
 * page at the same place race: lora_kv_plan gives every sequence a page of its own to write to.
 * A row of no sequence, or whose place is outside the table, or whose page is outside the cache is not
 * written (LORA_STATUS_BAD_LENGTH twice, LORA_STATUS_BAD_PAGE), its q is.  One launch.
 */
int lora_rope_append(const lora_kv_cache *cache, int layer, const lora_kv_batch *batch,
                     const lora_rope *rope, const void *q, int64_t ldq, const void *k, int64_t ldk,
                     const void *v, int64_t ldv, void *q_out, int64_t ldqo, int n_heads,
                     int in_dtype, void *stream);

/* ------------------------------------------------------------------------------------
 * Attention of the batch's new rows over the cache, which holds their own K and V already:
 *   out[t][h] = sum over visible j of softmax_j(scale * q[t][h] . K[j][h / g]) V[j][h / g],
 * g = n_heads / cache->n_heads (a whole number, 1 .. LORA_KV_MAX_GROUP).  Visible to the row at
 * position p are the tokens 0 <= j < seq_len, with causal != 0 only j <= p, with window > 0
 * (causal only) only j > p - window.  A row that sees nothing gives zeros.  q, out: bf16, row
 * strides ldq, ldo in elements, multiples of 8, not overlapping.  lse: device fp32
 * [n_rows][n_heads] or NULL, the natural logarithm of the sum of exp(scale * q . K), -inf for a
 * row that sees nothing.  n_rows * n_heads: at most 2^29 (LORA_ERR_TOO_LARGE).  scale: finite, > 0.
 * What pages hold past a sequence's length, and tokens that a row does not see, have no effect on it,
 * NaN and infinities included; an infinity or NaN of V that it does see makes that element of its
 * output infinite or NaN.  Scores, softmax sums and output sums are fp32, the softmax weights are
 * rounded to bf16 for the product with V.  Results are bit-identical run to run.  A length below zero
 * or beyond the table raises LORA_STATUS_BAD_LENGTH and is taken for the nearest that is not, a table
 * entry that is no page LORA_STATUS_BAD_PAGE; that sequence's rows mean nothing then.
 * ws: device scratch of lora_kv_attention_ws_bytes, which depends on the cache's heads, the
 * batch's n_seqs, n_rows and max_rows, and n_heads, not on lengths.
 * ------------------------------------------------------------------------------------ */
size_t lora_kv_attention_ws_bytes(const lora_kv_cache *cache, const lora_kv_batch *batch, int n_heads);

int lora_kv_attention(const lora_kv_cache *cache, int layer, const lora_kv_batch *batch,
                      const void *q, int64_t ldq, int n_heads, void *out, int64_t ldo, float *lse,
                      float scale, int causal, int window, void *ws, size_t ws_bytes, void *stream);

/* ------------------------------------------------------------------------------------
 * Pages.  A state says which pages the sequences in its n_seqs slots hold: the first
 * ceil(seq_len / page_size) entries of a slot's table row.  Slots may share pages (a common
 * prompt); page_ref counts the slots that hold a page, 0 = free.  Prefixes that outlive their
 * sequences are kept in slots of their own.
 *
 * lora_kv_plan turns one state into the next.  Slot s of `to` takes the first
 * min(seq_len[src[s]], new_len[s]) tokens of slot src[s] of `from` (src[s] = -1: none) and is as
 * long as new_len[s].  So s = src[s] with a larger new_len is growth, with a smaller one a fall
 * back, with 0 the end of a sequence; another slot's number is a fork.  Whole pages are shared.  A slot
 * that grows into a partly filled page that another slot of `to` holds too gets a page of its
 * own with the tokens so far (if all that hold the page grow into it, the lowest slot keeps
 * it).  Pages are taken lowest number first, in the order of the slots, for every slot first the
 * copy, then those it grows by.  `from` is only read, so kernels of the step before may still run
 * on it; its table and seq_len may not be `to`'s.  Table entries past a slot's pages become -1.
 *   counts = { pages in use, moves, free pages, pages asked for }
 * moves->pairs lists the copies (from, to), by slot.  A plan that asks for more pages than are
 * free, or whose lengths, sources or pages make no sense, raises its status bit and changes
 * nothing: `to` becomes `from` (page_ref only if `from` has one), without moves, and counts are
 * { 0, 0, 0, pages asked for } (0 as the last one too unless pages were all that was missing).
 *
 * lora_kv_compact: pages with numbers at or above the number of pages in use move, in order, to
 * the free numbers below it, and the tables follow.  Same counts, the last one 0.
 *
 * lora_kv_copy_pages moves the data of all layers as the pairs say.  Sources and destinations of
 * one list never overlap, so its copies run at once.  It has to run before the new state's pages
 * are written (lora_rope_append) or read.  max_moves: the host's bound on the number of pairs
 * (n_seqs after a plan, n_pages / 2 after a compaction), at most the list's capacity.
 * ------------------------------------------------------------------------------------ */
typedef struct lora_kv_state {
    int32_t n_seqs, max_pages;
    int32_t *table;       /* device [n_seqs][max_pages] */
    int32_t *seq_len;     /* device [n_seqs] */
    int32_t *page_ref;    /* device [n_pages of the cache]; NULL in `from` and `to` if not wanted */
} lora_kv_state;

typedef struct lora_kv_moves {
    int32_t capacity;     /* pairs that fit: n_seqs for a plan, n_pages / 2 for a compaction */
    int32_t reserved;
    int32_t *pairs;       /* device [capacity][2]: from, to */
    int32_t *counts;      /* device [4] */
    uint32_t *status;     /* device [1] */
    void *ws;             /* device scratch of lora_kv_moves_ws_bytes */
    size_t ws_bytes;
} lora_kv_moves;

size_t lora_kv_moves_ws_bytes(int n_pages, int n_seqs);

int lora_kv_plan(const lora_kv_cache *cache, const lora_kv_state *from, const lora_kv_state *to,
                 const int32_t *src, const int32_t *new_len, const lora_kv_moves *moves,
                 void *stream);

int lora_kv_compact(const lora_kv_cache *cache, const lora_kv_state *from, const lora_kv_state *to,
                    const lora_kv_moves *moves, void *stream);

int lora_kv_copy_pages(const lora_kv_cache *cache, const lora_kv_moves *moves, int max_moves,
                       void *stream);

#ifdef __cplusplus
}
#endif
#endif /* LORA_ATTN_H */
