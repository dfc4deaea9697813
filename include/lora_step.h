/*
 * What stands between the blocks of a step of an LLM instance whose adapters are served from a pool: the
 * residual's addition with the norm in front of the next products (whose rows lora_apply_group and lora_moe_apply take
 * as x), and the choice of the next tokens from the last product's logits.
 *
 * The conventions of lora.h hold: status codes and no exceptions, device memory owned by the caller, all work
 * on `stream` and nothing that waits, host-detectable mistakes before any device work.  Neither call needs a workspace.
 */
#ifndef LORA_STEP_H
#define LORA_STEP_H

#include "lora.h"

#ifdef __cplusplus
extern "C" {
#endif

enum {
    LORA_NORM_MAX_WIDTH = 65536,
    LORA_NORM_MAX_ROWS = 1 << 24,
    LORA_SAMPLE_MAX_VOCAB = 1 << 22
};

/* ------------------------------------------------------------------------------------
 * Residual and norm.  Row by row, in fp32:
 *   s = x + add,   r = 1 / sqrt(mean of s^2 + eps),   y = s * r * (weight + shift)
 * sum receives s, in x's type, out y in bf16, out8 y in 8 bits with scales (the product of a base weight in 8 bits takes
 * these, the adapters' products the bf16 rows); each is rounded once, to nearest even (values in 8 bits
 * from their quotient with the scale in fp32).  x_dtype, add_dtype and the weights'
 * dtype: LORA_DTYPE_BF16 or LORA_DTYPE_F32.  add NULL: s = x.  sum, out, out8: NULL if not wanted, one at least is.
 * Rows are row-major, their strides in elements and multiples of 8.  sum and out may be x or add itself where the element types
 * and strides are the same; other overlaps are not allowed.  Squares that are beyond fp32 are not lost: a row is scaled first if
 * their sum, or their mean with eps, is infinite.  A NaN or an infinity in s makes its row's y NaN, or 0 where only others are infinite.
 *
 * out8: values in e4m3 (4 exponent bits, 3 of mantissa, largest value 448, no infinities).  The columns of a row are cut into groups of
 * `group` (a power of two, 8 .. 512, the last group may be shorter; 0: the whole row); each has a scale, the largest |y| over 448,
 * or 1 if that is 0: y = value * scale up to the rounding of value.  scale[row * ld_scale + i] is that of group i.  A NaN in a group
 * makes its scale and values NaN.  Scales below 2^-126 are not exact.
 * ------------------------------------------------------------------------------------ */
typedef struct lora_norm {
    const void *weight;       /* device [width], 16-byte aligned, or NULL: ones */
    int32_t width;            /* a multiple of 8, 8 .. LORA_NORM_MAX_WIDTH */
    int32_t weight_dtype;
    float eps;                /* positive and normal */
    float shift;              /* finite; 1 where weights are held as differences from one */
} lora_norm;

typedef struct lora_rows8 {
    void *values;             /* device [n_rows][width], 16-byte aligned */
    float *scale;             /* device */
    int64_t ld;               /* of values: bytes, a multiple of 8 */
    int64_t ld_scale;         /* at least the number of groups */
    int32_t group;
    int32_t reserved;
} lora_rows8;

int lora_add_norm(const lora_norm *norm, int n_rows, const void *x, int64_t ldx, int x_dtype, const void *add,
                  int64_t ldadd, int add_dtype, void *sum, int64_t ldsum, void *out, int64_t ldo,
                  const lora_rows8 *out8, void *stream);

/* ------------------------------------------------------------------------------------
 * The next token of every row of logits, from one given random number each.  With l the logits of a row and T its
 * temperature, token i has the weight w_i = exp((l_i - max l) / T), and tokens stand in the order of falling l, equal ones by
 * number.  Kept are
 *   top_k   the first k of that order
 *   top_p   then, the fewest first ones whose weight reaches top_p times the weight of what top_k has left (one at least)
 *   min_p   of these, the ones with w >= min_p
 * and the token is the first one, by number, at which the sum of the kept weights up to it exceeds u times the sum of all kept.
 * T <= 0 or NaN: the first token of the order.  top_k <= 0, top_p >= 1 or NaN, min_p <= 0 or NaN: no such limit; min_p > 1 counts as 1.
 * u below 0 or NaN counts as 0, from 1 on as the largest number below.  A logit of -inf or NaN is never chosen; where a row has
 * no other the token is -1.  With logits of +inf, these have the weight 1 and all others none.
 * prob: the probability with which the token was chosen, its weight over the sum of the kept ones; 1 at T <= 0, 0 with token -1.
 *
 * Weights are formed in 64 bits and summed in whole multiples of 2^-46 (2^-(62 - b) for vocabularies of more than 2^16 tokens, b
 * the bits of their numbers), so that results do not depend on any order of additions; weights that round to zero are never chosen.
 * dtype: LORA_DTYPE_BF16 or LORA_DTYPE_F32.  ld: elements, at least vocab; logits need only be aligned to their type.
 * Columns behind the vocabulary are not read.
 * ------------------------------------------------------------------------------------ */
typedef struct lora_sampling {
    const float *temperature;   /* device [n_rows], NULL: 1 */
    const int32_t *top_k;       /* device [n_rows], NULL: no limit */
    const float *top_p;         /* device [n_rows], NULL: no limit */
    const float *min_p;         /* device [n_rows], NULL: no limit */
} lora_sampling;

int lora_sample(const void *logits, int64_t ld, int dtype, int n_rows, int vocab, const lora_sampling *how,
                const float *u, int32_t *token, float *prob, void *stream);

#ifdef __cplusplus
}
#endif
#endif /* LORA_STEP_H */
