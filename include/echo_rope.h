/*
 * echo_rope.h -- rotary positions (GPU).
 *
 * The first rotary_dim = R columns of a head [D] are R / 2 pairs, each turned by an
 * angle that grows with the token's position:
 *   (a, b) -> m * (a cos(p f_i) - b sin(p f_i), b cos(p f_i) + a sin(p f_i)),
 * pair i being columns i and i + R / 2 (ECHO_ROPE_HALF) or 2 i and 2 i + 1
 * (ECHO_ROPE_INTERLEAVED), f_i the pair's frequency in radians a position and m a
 * magnitude.  Columns from R on are copied.  Angles are reduced in 64 bits: their
 * error is below 2^-22 radians at any 32-bit position.
 *
 * The conventions of echo.h hold: device pointers on the current device, work
 * enqueued on `stream`, nothing allocated, nothing kept, every check before
 * anything is enqueued, status codes with a detail in echo_last_error().
 */
#ifndef ECHO_ROPE_H
#define ECHO_ROPE_H

#include <stddef.h>
#include <stdint.h>

#include "echo_fp8.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef enum { ECHO_ROPE_HALF = 0, ECHO_ROPE_INTERLEAVED = 1 } echo_rope_layout_t;

/* How frequencies f = theta^(-2 i / R) are scaled by s = factor for contexts longer
 * than those of training (L = original_length):
 *   NONE    f
 *   LINEAR  f / s: positions are interpolated
 *   NTK     theta is multiplied by s^(R / (R - 2)), which divides the last pair's
 *           frequency by s and leaves the first one's (R = 2: f)
 *   BANDS   by turns over the trained length, u = L f / (2 pi): f where u >= high, f / s
 *           where u <= low, between them f (m + (1 - m) / s), m = (u - low) / (high - low)
 *   YARN    by the pair's index: with d(u) = R ln(L / (2 pi u)) / (2 ln theta) the index
 *           of u turns, lo = max(floor(d(high)), 0), hi = min(ceil(d(low)), R - 1),
 *           f (m + (1 - m) / s), m = 1 - clamp((i - lo) / max(hi - lo, 0.001), 0, 1);
 *           the magnitude is 0.1 ln(s) + 1 */
typedef enum {
    ECHO_ROPE_NONE = 0,
    ECHO_ROPE_LINEAR = 1,
    ECHO_ROPE_NTK = 2,
    ECHO_ROPE_BANDS = 3,
    ECHO_ROPE_YARN = 4
} echo_rope_scaling_t;

typedef struct {
    int32_t head_dim;         /* D, at most 1024 */
    int32_t rotary_dim;       /* R, even, 2 to D */
    int32_t layout;           /* echo_rope_layout_t */
    int32_t scaling;          /* echo_rope_scaling_t */
    double theta;             /* above 0 (YARN: above 1), e.g. 500000 */
    double factor;            /* s >= 1 (not read under NONE) */
    double low, high;         /* turns, 0 < low < high (BANDS, YARN) */
    int32_t original_length;  /* L > 0 (BANDS, YARN) */
} echo_rope_t;

/* The R / 2 frequencies and the magnitude, in host memory (host only). */
int echo_rope_frequencies(const echo_rope_t *rope, double *frequencies, double *magnitude);

/* Heads [num_tokens][heads][D] of one tensor, in and out: tokens and heads any number
 * of elements apart (columns are adjacent).  out may be in itself with the same
 * strides, and overlaps it in no other way. */
typedef struct {
    const void *in;
    void *out;
    int32_t heads;
    int64_t in_token, in_head, out_token, out_head;
} echo_rope_heads_t;

/* Rotates the heads of one or two tensors (queries and keys) of `dtype` (echo_dtype_t).
 * Of `rope` head_dim, rotary_dim and layout are read.  frequencies: device fp64 [R / 2],
 * those of echo_rope_frequencies() or any others; positions: device int32 [num_tokens],
 * of either sign.  inverse: turned back (by -p f_i, still times the magnitude), which
 * is the gradient of the turn, and what takes a cached key to another position.  The
 * tensors do not overlap one another but for in and out of one. */
int echo_rope_rotate(const echo_rope_t *rope, const double *frequencies, double magnitude,
                     const int32_t *positions, int32_t num_tokens, int32_t dtype,
                     const echo_rope_heads_t *tensors, int32_t num_tensors, int32_t inverse,
                     void *stream);

#ifdef __cplusplus
}
#endif

#endif /* ECHO_ROPE_H */
