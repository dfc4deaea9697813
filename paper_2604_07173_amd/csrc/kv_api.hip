// C-ABI entry points of the paged cache: argument checks and launch parameters.  As in api.hip, every check
// that the host can make comes before the first HIP call.
#include <limits.h>
#include <string.h>

#include <algorithm>
#include <cmath>
#include <limits>

#include "kv_internal.h"
#include "kv_layout.h"
#include "kv_work.h"

using namespace lora;

namespace {

bool aligned(const void *p, size_t a) { return (reinterpret_cast<uintptr_t>(p) % a) == 0; }

#define LORA_HIP(expr)                                       \
    do {                                                     \
        hipError_t e_ = (expr);                              \
        if (e_ != hipSuccess) return note_hip_error(e_);     \
    } while (0)

int log2_of(int n)
{
    int s = 0;
    while ((1 << s) < n) ++s;
    return s;
}

constexpr int64_t kMaxExtent = (int64_t)1 << 61;      // elements: their bytes are counted in 63 bits too

// Elements from the first to the last of n things that lie `stride` apart and are `each` long, 0 if beyond kMaxExtent.
int64_t span(int64_t n, int64_t stride, int64_t each)
{
    int64_t far;
    return __builtin_mul_overflow(n - 1, stride, &far) || far > kMaxExtent - each ? 0 : far + each;
}

int check_cache(const lora_kv_cache *c)
{
    if (!c || !c->k || !c->v) return LORA_ERR_INVALID_ARG;
    if (!aligned(c->k, 16) || !aligned(c->v, 16)) return LORA_ERR_MISALIGNED;
    if (c->n_layers < 1 || c->n_pages < 1 || c->n_heads < 1) return LORA_ERR_INVALID_ARG;
    if (c->n_layers > 16384 || c->n_heads > 32768 || c->n_pages > LORA_KV_MAX_PAGES) return LORA_ERR_TOO_LARGE;
    if (c->page_size < 1 || c->page_size > LORA_KV_MAX_PAGE || (c->page_size & (c->page_size - 1))) return LORA_ERR_BAD_SHAPE;
    if (c->head_dim < 8 || c->head_dim > LORA_KV_MAX_HEAD_DIM || c->head_dim % 8) return LORA_ERR_BAD_SHAPE;
    const int64_t strides[4] = {c->layer_stride, c->page_stride, c->head_stride, c->token_stride};
    for (int64_t s : strides)
        if (s < 0 || s % 8 || s > ((int64_t)1 << 48)) return LORA_ERR_BAD_SHAPE;
    // each, in the order of the strides, begins beyond all that those with smaller ones span
    struct {
        int64_t n, stride;
    } dims[4] = {{c->n_layers, c->layer_stride}, {c->n_pages, c->page_stride}, {c->n_heads, c->head_stride}, {c->page_size, c->token_stride}};
    std::sort(dims, dims + 4, [](const auto &a, const auto &b) { return a.stride < b.stride; });
    int64_t extent = c->head_dim;
    for (const auto &d : dims) {
        if (d.n == 1) continue;
        if (d.stride < extent) return LORA_ERR_BAD_SHAPE;
        if (!(extent = span(d.n, d.stride, extent))) return LORA_ERR_TOO_LARGE;
    }
    return LORA_OK;
}

// with_cache: the call uses the tables
int check_batch(const lora_kv_batch *b, bool with_cache)
{
    if (!b) return LORA_ERR_INVALID_ARG;
    if (b->n_seqs < 0 || b->n_rows < 0 || b->max_rows < 0 || b->max_pages < 0) return LORA_ERR_INVALID_ARG;
    if (b->n_rows > LORA_MAX_ROWS_LONG || b->n_seqs > LORA_MAX_ROWS_LONG) return LORA_ERR_TOO_LARGE;
    if (b->n_rows == 0) return LORA_OK;
    if (!with_cache && b->position) return LORA_OK;
    if (b->n_seqs < 1 || !b->row_start || !b->seq_len) return LORA_ERR_INVALID_ARG;
    if (with_cache && (!b->table || b->max_pages < 1 || !b->status)) return LORA_ERR_INVALID_ARG;
    return LORA_OK;
}

int check_rows(const void *ptr, int64_t ld, int64_t width)
{
    if (!ptr) return LORA_ERR_INVALID_ARG;
    if (!aligned(ptr, 16)) return LORA_ERR_MISALIGNED;
    if (ld < width || ld % 8 || ld > ((int64_t)1 << 40)) return LORA_ERR_BAD_SHAPE;
    return LORA_OK;
}

KvView view_of(const lora_kv_cache *c, int layer)
{
    KvView v;
    v.k = static_cast<uint16_t *>(c->k) + layer * c->layer_stride;
    v.v = static_cast<uint16_t *>(c->v) + layer * c->layer_stride;
    v.page_stride = c->page_stride;
    v.head_stride = c->head_stride;
    v.token_stride = c->token_stride;
    v.n_pages = c->n_pages;
    v.page_shift = log2_of(c->page_size);
    v.n_heads = c->n_heads;
    v.dim = c->head_dim;
    return v;
}

KvRows rows_of(const lora_kv_batch *b, int page_size)
{
    KvRows r;
    r.row_start = b->row_start;
    r.seq_len = b->seq_len;
    r.table = b->table;
    r.position = b->position;
    r.status = b->status;
    r.n_seqs = b->n_seqs;
    r.n_rows = b->n_rows;
    r.max_pages = b->max_pages;
    const int64_t room = (int64_t)b->max_pages * page_size;
    r.tokens_max = (int)(room < (1 << 30) ? room : (1 << 30));     // offsets inside a sequence stay far below 2^31
    return r;
}

// What both calls of a batch with groups look at.
int check_shared(const lora_kv_shared *s, const lora_kv_batch *b)
{
    if (!s || s->n_seqs < 0 || s->n_rows < 0 || s->max_group_rows < 0) return LORA_ERR_INVALID_ARG;
    if (s->n_seqs > LORA_MAX_ROWS_LONG || s->n_rows > LORA_MAX_ROWS_LONG) return LORA_ERR_TOO_LARGE;
    if (b->n_rows == 0) return LORA_OK;
    if (!s->groups || !s->own || !s->place || !s->counts || (s->n_rows > 0 && !s->rows)) return LORA_ERR_INVALID_ARG;
    if (s->n_seqs != b->n_seqs) return LORA_ERR_BAD_SHAPE;
    return LORA_OK;
}

int check_attention(const void *q, int64_t ldq, const void *out, int64_t ldo, const float *lse, int64_t width, const void *ws)
{
    int rc;
    if ((rc = check_rows(q, ldq, width)) != LORA_OK) return rc;
    if ((rc = check_rows(out, ldo, width)) != LORA_OK) return rc;
    if (q == out || !ws) return LORA_ERR_INVALID_ARG;
    if (!aligned(ws, 16) || !aligned(lse, 4)) return LORA_ERR_MISALIGNED;
    return LORA_OK;
}

AttnParams attention_params(const lora_kv_cache *cache, int layer, const lora_kv_batch *batch, const void *q, int64_t ldq, int n_heads,
                            void *out, int64_t ldo, float *lse, float scale, int causal)
{
    AttnParams p;
    memset(&p, 0, sizeof p);
    p.c = view_of(cache, layer);
    p.b = rows_of(batch, cache->page_size);
    p.q = static_cast<const uint16_t *>(q);
    p.out = static_cast<uint16_t *>(out);
    p.lse = lse;
    p.ldq = ldq;
    p.ldo = ldo;
    // below infinity: equal scores stay equal, and all others are further apart than any weight shows
    p.scale_log2 = (float)std::min(scale * 1.4426950408889634, (double)std::numeric_limits<float>::max());
    p.heads = n_heads;
    p.group = n_heads / cache->n_heads;
    p.group_div = fast_div(p.group);
    p.kv_div = fast_div(cache->n_heads);
    p.heads_div = fast_div(n_heads);
    p.causal = causal != 0;
    return p;
}

int check_state(const lora_kv_state *s)
{
    if (!s || !s->table || !s->seq_len || s->n_seqs < 1 || s->max_pages < 1) return LORA_ERR_INVALID_ARG;
    if (s->n_seqs > LORA_MAX_ROWS_LONG) return LORA_ERR_TOO_LARGE;
    return LORA_OK;
}

int plan_params(const lora_kv_cache *cache, const lora_kv_state *from, const lora_kv_state *to,
                const lora_kv_moves *moves, int pairs, PlanParams &p)
{
    int rc = check_cache(cache);
    if (rc != LORA_OK) return rc;
    if ((rc = check_state(from)) != LORA_OK || (rc = check_state(to)) != LORA_OK) return rc;
    if (from->n_seqs != to->n_seqs || from->max_pages != to->max_pages) return LORA_ERR_BAD_SHAPE;
    if (from->table == to->table || from->seq_len == to->seq_len) return LORA_ERR_INVALID_ARG;
    if (to->page_ref && from->page_ref == to->page_ref) return LORA_ERR_INVALID_ARG;
    if (!moves || !moves->counts || !moves->status || !moves->ws || (pairs > 0 && !moves->pairs)) return LORA_ERR_INVALID_ARG;
    if (!aligned(moves->ws, 16)) return LORA_ERR_MISALIGNED;
    if (moves->capacity < pairs || moves->ws_bytes < plan_ws_bytes(cache->n_pages, from->n_seqs)) return LORA_ERR_BUFFER_TOO_SMALL;
    memset(&p, 0, sizeof p);
    p.from_table = from->table;
    p.from_len = from->seq_len;
    p.from_ref = from->page_ref;
    p.to_table = to->table;
    p.to_len = to->seq_len;
    p.to_ref = to->page_ref;
    p.pairs = moves->pairs;
    p.counts = moves->counts;
    p.status = moves->status;
    p.ws = static_cast<int32_t *>(moves->ws);
    p.n_pages = cache->n_pages;
    p.n_seqs = from->n_seqs;
    p.max_pages = from->max_pages;
    p.page_shift = log2_of(cache->page_size);
    return LORA_OK;
}

}  // namespace

extern "C" {

int lora_rope_freqs(const lora_rope_desc *d, double *freq)
{
    if (!d || !freq) return LORA_ERR_INVALID_ARG;
    if (d->rot_dim < 2 || d->rot_dim > LORA_KV_MAX_HEAD_DIM || d->rot_dim % 2) return LORA_ERR_BAD_SHAPE;
    if (!(d->base > 1.0) || !std::isfinite(d->base) || !(d->factor >= 1.0) || !std::isfinite(d->factor)) return LORA_ERR_INVALID_ARG;
    if (d->scaling < LORA_ROPE_PLAIN || d->scaling > LORA_ROPE_PARTS) return LORA_ERR_INVALID_ARG;
    if (d->scaling == LORA_ROPE_PARTS && (!(d->original_len > 0.0) || !std::isfinite(d->original_len) || !(d->low >= 0.0) ||
                                          !(d->high > d->low) || !std::isfinite(d->high)))
        return LORA_ERR_INVALID_ARG;
    const int rot = d->rot_dim;
    double base = d->base;
    if (d->scaling == LORA_ROPE_BASE && rot > 2) base *= std::pow(d->factor, rot / (rot - 2.0));
    for (int i = 0; i < rot / 2; ++i) {
        double f = std::pow(base, -2.0 * i / rot);
        if (d->scaling == LORA_ROPE_LINEAR) f /= d->factor;
        if (d->scaling == LORA_ROPE_PARTS) {
            const double turns = d->original_len * f / 6.283185307179586476925;
            double g = (turns - d->low) / (d->high - d->low);
            g = g < 0.0 ? 0.0 : g > 1.0 ? 1.0 : g;
            f = g * f + (1.0 - g) * f / d->factor;
        }
        freq[i] = f;
    }
    return LORA_OK;
}

int lora_rope_append(const lora_kv_cache *cache, int layer, const lora_kv_batch *batch, const lora_rope *rope,
                     const void *q, int64_t ldq, const void *k, int64_t ldk, const void *v, int64_t ldv, void *q_out,
                     int64_t ldqo, int n_heads, int in_dtype, void *stream)
{
    int rc = check_cache(cache);
    if (rc != LORA_OK) return rc;
    if (layer < 0 || layer >= cache->n_layers) return LORA_ERR_BAD_SHAPE;
    if (in_dtype != LORA_DTYPE_BF16 && in_dtype != LORA_DTYPE_F32) return LORA_ERR_INVALID_ARG;
    if (!k != !v || (!q && !k)) return LORA_ERR_INVALID_ARG;
    rc = check_batch(batch, k != nullptr);
    if (rc != LORA_OK) return rc;
    const int64_t D = cache->head_dim;
    if (q) {
        if (n_heads < 1 || n_heads > 32768) return LORA_ERR_BAD_SHAPE;
        if (batch->n_rows > 0) {
            if ((rc = check_rows(q, ldq, n_heads * D)) != LORA_OK) return rc;
            if ((rc = check_rows(q_out, ldqo, n_heads * D)) != LORA_OK) return rc;
            if (q == q_out && (in_dtype != LORA_DTYPE_BF16 || ldq != ldqo)) return LORA_ERR_INVALID_ARG;
        }
    }
    if (k && batch->n_rows > 0) {
        if ((rc = check_rows(k, ldk, cache->n_heads * D)) != LORA_OK) return rc;
        if ((rc = check_rows(v, ldv, cache->n_heads * D)) != LORA_OK) return rc;
    }
    if (rope) {
        if (!rope->freq) return LORA_ERR_INVALID_ARG;
        if (!aligned(rope->freq, 8)) return LORA_ERR_MISALIGNED;
        if (rope->rot_dim < 2 || rope->rot_dim % 2 || rope->rot_dim > D) return LORA_ERR_BAD_SHAPE;
        if (rope->pairing != LORA_ROPE_HALF && rope->pairing != LORA_ROPE_INTERLEAVED) return LORA_ERR_INVALID_ARG;
        if (!std::isfinite(rope->amplitude)) return LORA_ERR_INVALID_ARG;
    }
    if (batch->n_rows == 0) return LORA_OK;
    AppendParams p;
    memset(&p, 0, sizeof p);
    p.c = view_of(cache, layer);
    p.b = rows_of(batch, cache->page_size);
    p.q = q;
    p.k = k;
    p.v = v;
    p.ldq = ldq;
    p.ldk = ldk;
    p.ldv = ldv;
    p.ldqo = ldqo;
    p.q_out = static_cast<uint16_t *>(q_out);
    p.heads = q ? n_heads : 0;
    p.kv_heads = k ? cache->n_heads : 0;
    p.f32 = in_dtype == LORA_DTYPE_F32;
    if (rope) {
        p.freq = rope->freq;
        p.amplitude = rope->amplitude;
        p.rot = rope->rot_dim;
        p.pairing = rope->pairing;
    }
    LORA_HIP(launch_append(p, static_cast<hipStream_t>(stream)));
    return LORA_OK;
}

size_t lora_kv_attention_ws_bytes(const lora_kv_cache *cache, const lora_kv_batch *batch, int n_heads)
{
    if (check_cache(cache) != LORA_OK || !batch || batch->n_seqs < 0 || batch->n_rows < 0 || batch->max_rows < 0) return 0;
    if (batch->n_rows > LORA_MAX_ROWS_LONG || batch->n_seqs > LORA_MAX_ROWS_LONG) return 0;
    if (n_heads < 1 || n_heads % cache->n_heads || n_heads / cache->n_heads > LORA_KV_MAX_GROUP) return 0;
    return attention_ws_bytes(batch->n_seqs, batch->n_rows, batch->max_rows, n_heads, cache->n_heads, cache->head_dim);
}

int lora_kv_attention(const lora_kv_cache *cache, int layer, const lora_kv_batch *batch, const void *q, int64_t ldq,
                      int n_heads, void *out, int64_t ldo, float *lse, float scale, int causal, int window, void *ws,
                      size_t ws_bytes, void *stream)
{
    int rc = check_cache(cache);
    if (rc != LORA_OK) return rc;
    if (layer < 0 || layer >= cache->n_layers) return LORA_ERR_BAD_SHAPE;
    rc = check_batch(batch, true);
    if (rc != LORA_OK) return rc;
    if (n_heads < 1 || n_heads % cache->n_heads || n_heads / cache->n_heads > LORA_KV_MAX_GROUP) return LORA_ERR_BAD_SHAPE;
    if (!std::isfinite(scale) || scale <= 0.f || window < 0 || (window > 0 && !causal)) return LORA_ERR_INVALID_ARG;
    if (batch->n_rows == 0) return LORA_OK;
    if ((int64_t)batch->n_rows * n_heads > (1 << 29)) return LORA_ERR_TOO_LARGE;
    const int64_t width = (int64_t)n_heads * cache->head_dim;
    if ((rc = check_attention(q, ldq, out, ldo, lse, width, ws)) != LORA_OK) return rc;
    if (ws_bytes < lora_kv_attention_ws_bytes(cache, batch, n_heads)) return LORA_ERR_BUFFER_TOO_SMALL;
    AttnParams p = attention_params(cache, layer, batch, q, ldq, n_heads, out, ldo, lse, scale, causal);
    p.window = window < p.b.tokens_max ? window : 0;     // as wide as the longest sequence: no window
    LORA_HIP(launch_attention(p, batch->max_rows, ws, static_cast<hipStream_t>(stream)));
    return LORA_OK;
}

size_t lora_kv_share_ws_bytes(int n_seqs)
{
    return n_seqs < 1 || n_seqs > LORA_MAX_ROWS_LONG ? 0 : share_ws_bytes(n_seqs);
}

int lora_kv_share(const lora_kv_cache *cache, const lora_kv_batch *batch, const lora_kv_shared *shared, int min_pages, int max_rows,
                  void *stream)
{
    int rc = check_cache(cache);
    if (rc != LORA_OK) return rc;
    if ((rc = check_batch(batch, true)) != LORA_OK) return rc;
    if ((rc = check_shared(shared, batch)) != LORA_OK) return rc;
    if (min_pages < 1 || max_rows < 0) return LORA_ERR_INVALID_ARG;
    if (batch->n_rows == 0) return LORA_OK;
    if (!shared->ws) return LORA_ERR_INVALID_ARG;
    if (!aligned(shared->ws, 16)) return LORA_ERR_MISALIGNED;
    const int64_t rows = max_rows ? std::min<int64_t>(batch->n_rows, (int64_t)batch->n_seqs * max_rows) : batch->n_rows;
    if (shared->n_rows < rows || shared->ws_bytes < share_ws_bytes(batch->n_seqs)) return LORA_ERR_BUFFER_TOO_SMALL;
    ShareParams p;
    memset(&p, 0, sizeof p);
    p.b = rows_of(batch, cache->page_size);
    p.groups = shared->groups;
    p.rows = shared->rows;
    p.own = shared->own;
    p.place = shared->place;
    p.counts = shared->counts;
    p.ws = static_cast<int32_t *>(shared->ws);
    p.page_shift = log2_of(cache->page_size);
    p.min_pages = min_pages;
    p.max_rows = max_rows ? max_rows : INT_MAX;
    p.most = groups_of(shared->n_seqs);
    p.most_rows = shared->n_rows;
    LORA_HIP(launch_share(p, static_cast<hipStream_t>(stream)));
    return LORA_OK;
}

size_t lora_kv_attention_shared_ws_bytes(const lora_kv_cache *cache, const lora_kv_batch *batch, const lora_kv_shared *shared, int n_heads)
{
    if (lora_kv_attention_ws_bytes(cache, batch, n_heads) == 0 || !shared || shared->n_rows < 0 || shared->n_rows > LORA_MAX_ROWS_LONG ||
        shared->max_group_rows < 0 || std::max(batch->n_rows, shared->n_rows) * (int64_t)n_heads > kSharedRowsHeads)
        return 0;
    return attention_shared_ws_bytes(batch->n_seqs, batch->n_rows, batch->max_rows, shared->n_rows, shared->max_group_rows, n_heads,
                                     cache->n_heads, cache->head_dim);
}

int lora_kv_attention_shared(const lora_kv_cache *cache, int layer, const lora_kv_batch *batch, const lora_kv_shared *shared,
                             const void *q, int64_t ldq, int n_heads, void *out, int64_t ldo, float *lse, float scale, int causal,
                             void *ws, size_t ws_bytes, void *stream)
{
    int rc = check_cache(cache);
    if (rc != LORA_OK) return rc;
    if (layer < 0 || layer >= cache->n_layers) return LORA_ERR_BAD_SHAPE;
    if ((rc = check_batch(batch, true)) != LORA_OK) return rc;
    if ((rc = check_shared(shared, batch)) != LORA_OK) return rc;
    if (n_heads < 1 || n_heads % cache->n_heads || n_heads / cache->n_heads > LORA_KV_MAX_GROUP) return LORA_ERR_BAD_SHAPE;
    if (!std::isfinite(scale) || scale <= 0.f) return LORA_ERR_INVALID_ARG;
    if (batch->n_rows == 0) return LORA_OK;
    if (std::max(batch->n_rows, shared->n_rows) * (int64_t)n_heads > kSharedRowsHeads) return LORA_ERR_TOO_LARGE;
    if ((rc = check_attention(q, ldq, out, ldo, lse, (int64_t)n_heads * cache->head_dim, ws)) != LORA_OK) return rc;
    if (ws_bytes < lora_kv_attention_shared_ws_bytes(cache, batch, shared, n_heads)) return LORA_ERR_BUFFER_TOO_SMALL;
    AttnParams p = attention_params(cache, layer, batch, q, ldq, n_heads, out, ldo, lse, scale, causal);
    p.g.groups = shared->groups;
    p.g.rows = shared->rows;
    p.g.own = shared->own;
    p.g.place = shared->place;
    p.g.counts = shared->counts;
    p.g.most = groups_of(shared->n_seqs);
    p.g.most_rows = shared->n_rows;
    LORA_HIP(launch_attention_shared(p, batch->max_rows, shared->max_group_rows, ws, static_cast<hipStream_t>(stream)));
    return LORA_OK;
}

size_t lora_kv_moves_ws_bytes(int n_pages, int n_seqs)
{
    if (n_pages < 1 || n_pages > LORA_KV_MAX_PAGES || n_seqs < 1 || n_seqs > LORA_MAX_ROWS_LONG) return 0;
    return plan_ws_bytes(n_pages, n_seqs);
}

int lora_kv_plan(const lora_kv_cache *cache, const lora_kv_state *from, const lora_kv_state *to, const int32_t *src,
                 const int32_t *new_len, const lora_kv_moves *moves, void *stream)
{
    PlanParams p;
    const int rc = plan_params(cache, from, to, moves, to ? to->n_seqs : 0, p);
    if (rc != LORA_OK) return rc;
    if (!src || !new_len) return LORA_ERR_INVALID_ARG;
    p.src = src;
    p.new_len = new_len;
    LORA_HIP(launch_plan(p, static_cast<hipStream_t>(stream)));
    return LORA_OK;
}

int lora_kv_compact(const lora_kv_cache *cache, const lora_kv_state *from, const lora_kv_state *to,
                    const lora_kv_moves *moves, void *stream)
{
    PlanParams p;
    const int rc = plan_params(cache, from, to, moves, cache ? cache->n_pages / 2 : 0, p);
    if (rc != LORA_OK) return rc;
    LORA_HIP(launch_compact(p, static_cast<hipStream_t>(stream)));
    return LORA_OK;
}

int lora_kv_copy_pages(const lora_kv_cache *cache, const lora_kv_moves *moves, int max_moves, void *stream)
{
    const int rc = check_cache(cache);
    if (rc != LORA_OK) return rc;
    if (!moves || !moves->counts || max_moves < 0 || (max_moves > 0 && !moves->pairs)) return LORA_ERR_INVALID_ARG;
    if (max_moves > moves->capacity) return LORA_ERR_BUFFER_TOO_SMALL;
    if (max_moves == 0) return LORA_OK;
    CopyParams p;
    memset(&p, 0, sizeof p);
    p.k = static_cast<uint16_t *>(cache->k);
    p.v = static_cast<uint16_t *>(cache->v);
    p.pairs = moves->pairs;
    p.counts = moves->counts;
    p.layer_stride = cache->layer_stride;
    p.page_stride = cache->page_stride;
    const PageRuns r = page_runs(*cache);
    p.run = r.run;
    p.inner = r.inner;
    p.outer = r.outer;
    p.inner_stride = r.inner_stride;
    p.outer_stride = r.outer_stride;
    p.run_vecs = fast_div(p.run / 8);
    p.inner_div = fast_div(p.inner);
    p.n_layers = cache->n_layers;
    p.n_pages = cache->n_pages;
    p.max_moves = max_moves;
    LORA_HIP(launch_copy_pages(p, static_cast<hipStream_t>(stream)));
    return LORA_OK;
}

}  // extern "C"
