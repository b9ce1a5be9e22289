/*
 * echo_norm.h -- what stands between two blocks of a decoder layer (GPU).
 *
 * In one pass over a token's row of H values:
 *   v   = post(block)                      the norm behind a block, if any
 *   sum = residual_scale * residual + block_scale * gate * v
 *   y   = pre(sum)                         the norm before the next block
 * with post and pre each one of
 *   NONE   x
 *   RMS    x / sqrt(mean(x^2) + eps) * weight (+ bias)
 *   LAYER  (x - mean(x)) / sqrt(mean((x - mean(x))^2) + eps) * weight (+ bias).
 * Rows are held in fp32 from the first to the last step: y is the norm of the sum
 * before it is rounded to its type.  A norm's squares and mean may leave fp32's range
 * where its input does not (rows above 1e19, or below 1e-19 without eps): such rows are
 * taken times a power of two.  An infinity makes a LAYER norm's row NaN; of an RMS norm's
 * row it leaves 0, and NaN in its own column.  Where y is int8 codes they are those of
 * echo_int8.h's rule for y in 64 bits (scale = fp32(amax / 127), 1 where that is 0,
 * code = y / scale to the nearest integer), and every step is taken in 64 bits, so
 * that codes hang on the order of sums only within 2^-40 steps of a border.  That order
 * goes by H alone where y is no codes: a row's results are the same in any batch.  Where it
 * is, it goes by the number of rows as well (up to 512 and more), and sum, rounded from 64
 * bits, may be a unit in the last place apart now and then.
 *
 * The conventions of echo.h hold: device pointers on the current device, work
 * enqueued on `stream`, nothing allocated, nothing kept, every check before
 * anything is enqueued, status codes with a detail in echo_last_error().
 */
#ifndef ECHO_NORM_H
#define ECHO_NORM_H

#include <stddef.h>
#include <stdint.h>

#include "echo_fp8.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef enum { ECHO_NORM_NONE = 0, ECHO_NORM_RMS = 1, ECHO_NORM_LAYER = 2 } echo_norm_kind_t;

/* Beside echo_dtype_t: int8 codes (of y only) */
enum { ECHO_I8 = 2 };

typedef struct {
    int32_t hidden;        /* H, 1 to 32768 (codes: to 16384) */
    int32_t post, pre;     /* echo_norm_kind_t */
    int32_t param_dtype;   /* ECHO_BF16 or ECHO_F32: of weights and biases [H] */
    float post_eps, pre_eps;
    float residual_scale, block_scale;
    float weight_offset;   /* added to every weight (1 where w - 1 is stored) */
    const void *post_weight, *post_bias;   /* may be NULL: weight + offset = 1, bias 0; */
    const void *pre_weight, *pre_bias;     /* not read where the norm is NONE */
} echo_norm_t;

/* Rows [num_tokens][H], stride elements apart.  data NULL: there is none. */
typedef struct {
    void *data;
    int32_t dtype;
    int64_t stride;
} echo_rows_t;

/* One pass for num_tokens rows.
 *   block     bf16 or fp32; none: sum = residual_scale * residual (gate not read)
 *   residual  bf16 or fp32; none: sum = block_scale * gate * v
 *             (one of block and residual is there)
 *   gate      bf16 or fp32; none: 1; stride 0: one row for every token
 *   sum       bf16 or fp32; none: not stored
 *   y         bf16, fp32 or int8 codes with scales y_scale [num_tokens] (not read
 *             otherwise); none: not computed.  A row of y with a NaN or an infinity
 *             has the scale NaN and codes of 0.
 *             (one of sum and y is there)
 * sum may be residual or block itself, y block or residual, each of its type and stride
 * (sum and y are two buffers); buffers overlap in no other way. */
int echo_norm_join(const echo_norm_t *norm, int32_t num_tokens, const echo_rows_t *block,
                   const echo_rows_t *gate, const echo_rows_t *residual, const echo_rows_t *sum,
                   const echo_rows_t *y, float *y_scale, void *stream);

#ifdef __cplusplus
}
#endif

#endif /* ECHO_NORM_H */
