/*
 * echo_moe.h -- experts in the place of a decoder layer's MLP (GPU).
 *
 * Each token goes through top_k of num_experts MLPs of the layer's form
 * (SiLU(x W_gate^T) * (x W_up^T)) W_down^T, chosen by a router.  Weights and
 * activations are e4m3 codes with scales (echo_fp8.h), whose conventions hold.
 */
#ifndef ECHO_MOE_H
#define ECHO_MOE_H

#include <stddef.h>
#include <stdint.h>

#include "echo_fp8.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef enum { ECHO_SCORE_SOFTMAX = 0, ECHO_SCORE_SIGMOID = 1 } echo_score_t;

/* How tokens choose experts. */
typedef struct {
    int32_t num_experts;   /* E, 1..512 */
    int32_t top_k;         /* experts of a token, 1..64, at most top_groups * E / num_groups */
    int32_t score;         /* echo_score_t */
    int32_t num_groups;    /* groups of E / num_groups consecutive experts, 1..64 */
    int32_t top_groups;    /* groups a token's experts may come from, 1..num_groups */
    int32_t group_top;     /* a group's score: the sum of its best 1 or 2 keys (2: at least
                              two experts a group) */
    int32_t renormalize;   /* nonzero: divide the weights by their sum */
    float scale;           /* factor of every weight, finite */
} echo_router_t;

/* For every token, from its logits [E] (bf16 or fp32, rows logits_stride >= E
 * elements apart), in 64 bits:
 *   score = softmax or sigmoid of the logits;
 *   key   = score + bias (bias: fp32 [E], optional: balances the experts
 *           without entering the weights), or the logit itself without a bias
 *           (a group's sum of two is of scores then), which orders as the score;
 *   the top_groups groups of the highest score are kept, then the top_k experts
 *   of the highest key in them; among equals the lowest index wins;
 *   ids [T][top_k] in falling order of key, weights [T][top_k] = score, over
 *   the sum of the chosen ones' scores with renormalize (0 where that is 0),
 *   times scale, rounded once.
 * A logit of NaN or -inf, or a key of NaN or -inf, is an expert that cannot be
 * chosen (and outside the softmax where the logit says so); +inf counts as the
 * largest finite value.  Where fewer than top_k experts can be chosen the rest
 * of the row has id -1 and weight 0, which echo_moe_experts skips. */
int echo_moe_route(const echo_router_t *router, const void *logits, int32_t logits_dtype,
                   int64_t logits_stride, int32_t num_tokens, const float *bias, int32_t *ids,
                   float *weights, void *stream);

/* The experts' weights: codes and their scales of 128 x 128 blocks, each matrix
 * (gate, up and down of each expert) in blocks of its own.  IB, HB =
 * ceil(I / 128), ceil(H / 128). */
typedef struct {
    int32_t num_experts;           /* E, 1..512 */
    int32_t hidden;                /* H, a multiple of 16 */
    int32_t intermediate;          /* I, a multiple of 16, at most 2^23 */
    const void *w_gate_up;         /* [E][2 I][H]: gate rows, then up rows */
    const float *gate_up_scale;    /* [E][2][IB][HB] */
    const void *w_down;            /* [E][H][I] */
    const float *down_scale;       /* [E][HB][IB] */
} echo_experts_t;

/* out[t] = (residual[t] +) sum_j weights[t][j] * expert(ids[t][j])(x[t]):
 * x codes [T][H] with scales of 1 x 128 (echo_fp8_quantize), ids and weights
 * [T][top_k], residual (optional; may be out itself) and out bf16 [T][H].
 * Inside an expert the activation SiLU(gate) * up, in fp32 (both products' sums are
 * as exact as echo_fp8_gemm's under a bf16 result, or better), is requantised in blocks of
 * 1 x 128 as echo_fp8_quantize does (quotients within two ulps); an expert's output
 * is rounded to 11 bits (2^-11 of the value, or 2^-39 of the largest of its 16 or
 * more neighbours) before the weighted sum, which is taken in fp32 in the order of
 * j.  A pair whose id lies outside [0, E) adds nothing, whatever its weight:
 * padding, or experts held elsewhere.  An expert may stand twice in a row.
 * T * top_k at most 2^24; top_k 1..64; T * H and 2 I H below 2^32.
 * Same inputs give the same bits.  workspace: as for echo_fp8_gemm, of
 * echo_moe_experts_workspace_bytes() bytes. */
int echo_moe_experts(const echo_experts_t *experts, const void *x, const float *x_scale,
                     int32_t num_tokens, int32_t top_k, const int32_t *ids, const float *weights,
                     const void *residual, void *out, void *workspace, size_t workspace_bytes,
                     void *stream);

/* Workspace bytes echo_moe_experts needs (0 and a detail in echo_last_error()
 * when the arguments are invalid; 0 for no tokens).  They do not fall with
 * num_tokens. */
size_t echo_moe_experts_workspace_bytes(const echo_experts_t *experts, int32_t num_tokens,
                                        int32_t top_k);

#ifdef __cplusplus
}
#endif

#endif /* ECHO_MOE_H */
