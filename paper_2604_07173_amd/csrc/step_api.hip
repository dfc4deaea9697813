// C-ABI entry points of the residual norm and of sampling: argument checks and launch parameters.  As in api.hip, every check that
// the host can make comes before the first HIP call.
#include <string.h>

#include <algorithm>
#include <cmath>

#include "step_internal.h"

using namespace lora;

namespace {

bool aligned(const void *p, size_t a) { return (reinterpret_cast<uintptr_t>(p) % a) == 0; }

#define LORA_HIP(expr)                                       \
    do {                                                     \
        hipError_t e_ = (expr);                              \
        if (e_ != hipSuccess) return note_hip_error(e_);     \
    } while (0)

bool is_dtype(int d) { return d == LORA_DTYPE_BF16 || d == LORA_DTYPE_F32; }

constexpr int64_t kMaxStride = (int64_t)1 << 36;      // elements: 2^24 rows of them are counted in 63 bits of bytes

int check_rows(const void *ptr, int64_t ld, int64_t width)
{
    if (!aligned(ptr, 16)) return LORA_ERR_MISALIGNED;
    if (ld < width || ld % 8 || ld > kMaxStride) return LORA_ERR_BAD_SHAPE;
    return LORA_OK;
}

// An output may be an input itself, element on element.
bool in_place(const void *out, int64_t ldo, int out_dtype, const void *in, int64_t ldi, int in_dtype)
{
    return out != in || (ldo == ldi && out_dtype == in_dtype);
}

}  // namespace

extern "C" {

int lora_add_norm(const lora_norm *norm, int n_rows, const void *x, int64_t ldx, int x_dtype, const void *add, int64_t ldadd,
                  int add_dtype, void *sum, int64_t ldsum, void *out, int64_t ldo, const lora_rows8 *out8, void *stream)
{
    if (!norm || n_rows < 0 || !is_dtype(x_dtype) || !is_dtype(norm->weight_dtype) || (add && !is_dtype(add_dtype))) return LORA_ERR_INVALID_ARG;
    if (norm->width < 8 || norm->width % 8) return LORA_ERR_BAD_SHAPE;
    if (norm->width > LORA_NORM_MAX_WIDTH || n_rows > LORA_NORM_MAX_ROWS) return LORA_ERR_TOO_LARGE;
    if (!std::isnormal(norm->eps) || norm->eps < 0.f || !std::isfinite(norm->shift)) return LORA_ERR_INVALID_ARG;
    if (!aligned(norm->weight, 16)) return LORA_ERR_MISALIGNED;
    if (!sum && !out && !out8) return LORA_ERR_INVALID_ARG;
    const int width = norm->width;
    if (out8) {
        const int g = out8->group;
        if (g != 0 && (g < 8 || g > 512 || (g & (g - 1)))) return LORA_ERR_BAD_SHAPE;
    }
    if (n_rows == 0) return LORA_OK;
    int rc;
    if (!x) return LORA_ERR_INVALID_ARG;
    if ((rc = check_rows(x, ldx, width)) != LORA_OK) return rc;
    if (add && (rc = check_rows(add, ldadd, width)) != LORA_OK) return rc;
    if (sum && (rc = check_rows(sum, ldsum, width)) != LORA_OK) return rc;
    if (out && (rc = check_rows(out, ldo, width)) != LORA_OK) return rc;
    if (sum && sum == out) return LORA_ERR_INVALID_ARG;
    if (sum && (!in_place(sum, ldsum, x_dtype, x, ldx, x_dtype) || !in_place(sum, ldsum, x_dtype, add, ldadd, add_dtype))) return LORA_ERR_INVALID_ARG;
    if (out && (!in_place(out, ldo, LORA_DTYPE_BF16, x, ldx, x_dtype) || !in_place(out, ldo, LORA_DTYPE_BF16, add, ldadd, add_dtype)))
        return LORA_ERR_INVALID_ARG;
    NormParams p;
    memset(&p, 0, sizeof p);
    if (out8) {
        if (!out8->values || !out8->scale) return LORA_ERR_INVALID_ARG;
        if (!aligned(out8->scale, 4)) return LORA_ERR_MISALIGNED;
        if ((rc = check_rows(out8->values, out8->ld, width)) != LORA_OK) return rc;
        const int groups = out8->group ? (width + out8->group - 1) / out8->group : 1;
        if (out8->ld_scale < groups || out8->ld_scale > kMaxStride) return LORA_ERR_BAD_SHAPE;
        if (out8->values == x || out8->values == add || out8->values == sum || out8->values == out) return LORA_ERR_INVALID_ARG;
        p.out8 = static_cast<uint8_t *>(out8->values);
        p.scale = out8->scale;
        p.ld8 = out8->ld;
        p.ld_scale = out8->ld_scale;
        p.group = out8->group;
    }
    p.x = x;
    p.add = add;
    p.weight = norm->weight;
    p.sum = sum;
    p.out = static_cast<uint16_t *>(out);
    p.ldx = ldx;
    p.ldadd = ldadd;
    p.ldsum = ldsum;
    p.ldo = ldo;
    p.n_rows = n_rows;
    p.width = width;
    p.weight_f32 = norm->weight_dtype == LORA_DTYPE_F32;
    p.eps = norm->eps;
    p.shift = norm->shift;
    LORA_HIP(launch_norm(p, x_dtype == LORA_DTYPE_F32, add_dtype == LORA_DTYPE_F32, static_cast<hipStream_t>(stream)));
    return LORA_OK;
}

int lora_sample(const void *logits, int64_t ld, int dtype, int n_rows, int vocab, const lora_sampling *how, const float *u,
                int32_t *token, float *prob, void *stream)
{
    if (!how || !is_dtype(dtype) || n_rows < 0) return LORA_ERR_INVALID_ARG;
    if (vocab < 1 || ld < vocab || ld > kMaxStride) return LORA_ERR_BAD_SHAPE;
    if (vocab > LORA_SAMPLE_MAX_VOCAB || n_rows > LORA_MAX_ROWS_LONG) return LORA_ERR_TOO_LARGE;
    if (n_rows == 0) return LORA_OK;
    if (!logits || !u || !token) return LORA_ERR_INVALID_ARG;
    if (!aligned(logits, dtype == LORA_DTYPE_F32 ? 4 : 2)) return LORA_ERR_MISALIGNED;
    for (const void *a : {(const void *)u, (const void *)token, (const void *)prob, (const void *)how->temperature, (const void *)how->top_k,
                          (const void *)how->top_p, (const void *)how->min_p})
        if (!aligned(a, 4)) return LORA_ERR_MISALIGNED;
    SampleParams p;
    memset(&p, 0, sizeof p);
    p.logits = logits;
    p.ld = ld;
    p.n_rows = n_rows;
    p.vocab = vocab;
    p.temperature = how->temperature;
    p.top_k = how->top_k;
    p.top_p = how->top_p;
    p.min_p = how->min_p;
    p.u = u;
    p.token = token;
    p.prob = prob;
    int bits = 0;
    while ((1 << bits) < vocab) ++bits;
    p.shift = std::min(46, 62 - bits);
    LORA_HIP(launch_sample(p, dtype == LORA_DTYPE_F32, static_cast<hipStream_t>(stream)));
    return LORA_OK;
}

}  // extern "C"
