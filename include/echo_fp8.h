/*
 * echo_fp8.h -- linear layers in 8-bit floating point (GPU).
 *
 * The decoder layer's products on operands held as OCP e4m3fn codes with one
 * fp32 scale per block of 128: activations in blocks of 1 x 128 (one row, 128
 * columns), weights in blocks of 128 x 128.  The value of a code is
 * e4m3(code) * scale of its block.  Blocks at the right and lower edges are
 * cut off; a matrix [rows][cols] has ceil(rows / block_rows) x ceil(cols / 128)
 * scales, row-major.
 *
 * The conventions of echo.h hold: device pointers on the current device, work
 * enqueued on `stream`, nothing allocated, nothing kept, every check before
 * anything is enqueued, status codes with a detail in echo_last_error().
 * Tensors are row-major; strides are in elements.  A call of no rows returns
 * ECHO_OK and touches nothing (its pointers may be NULL).
 */
#ifndef ECHO_FP8_H
#define ECHO_FP8_H

#include <stddef.h>
#include <stdint.h>

#include "echo.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef enum { ECHO_BF16 = 0, ECHO_F32 = 1 } echo_dtype_t;

/* Codes and scales of `batch` stacked matrices x [rows][cols] (bf16 or fp32,
 * rows x_stride elements apart, matrices rows * x_stride apart), in blocks of
 * block_rows x 128, block_rows 1 (activations) or 128 (weights):
 *   scale = fp32(amax / 448) over the block, 1 where that is 0;
 *   code  = the round-to-nearest-even e4m3 encoding, saturating at 448, of the
 *           correctly rounded fp32 quotient x / scale,
 * the rule of e4m3 cache blocks (echo_kv_append).  A NaN keeps out of amax and
 * gets the NaN code; a block with an infinity gets the scale infinity, codes 0
 * for its finite values and the NaN code for the infinities.
 * codes: [batch][rows][cols]; scales: [batch][ceil(rows / block_rows)]
 * [ceil(cols / 128)].  cols a multiple of 16; x and codes 16-byte aligned, and
 * x_stride >= cols with rows at 16-byte steps.  The buffers do not overlap. */
int echo_fp8_quantize(const void *x, int32_t x_dtype, int64_t x_stride, int32_t batch,
                      int32_t rows, int32_t cols, int32_t block_rows, void *codes, float *scales,
                      void *stream);

/* y[t][n] = sum_b x_scale[t][b] * w_scale[n / 128][b] * sum_{k in block b} x[t][k] w[n][k]
 *           (+ residual[t][n]),
 * x codes [T][K] with scales of 1 x 128, w codes [N][K] (out_features x
 * in_features) with scales of 128 x 128, sums in fp32, y [T][N] bf16 or fp32
 * with rows y_stride >= N elements apart, rounded once.  An fp32 result takes
 * exact products and fp32 sums; under a bf16 result the e4m3 matrix instructions add
 * products, those of eight neighbours along K cut off towards zero at 2^-13 of the
 * largest: 1.5e-5 of the sum in the 2-norm where terms are of both signs and alike,
 * 7 x 2^-13 of the largest of every eight at worst.  Scales may be any fp32 numbers: it is
 * the scaled sum of a block that has to be one, not the product of its scales.
 * residual (optional):
 * of y's type and strides, added before that rounding; it may be y itself, and
 * overlaps it in no other way; y overlaps no other buffer.  K a multiple of 16,
 * at most 2^23; x and w 16-byte aligned.
 * workspace: device scratch of echo_fp8_gemm_workspace_bytes() bytes (may be
 * none), 256-byte aligned, used by no other call until this one has completed. */
int echo_fp8_gemm(const void *x, const float *x_scale, const void *w, const float *w_scale,
                  int32_t num_tokens, int32_t out_features, int32_t in_features,
                  const void *residual, void *y, int32_t y_dtype, int64_t y_stride,
                  void *workspace, size_t workspace_bytes, void *stream);

/* Workspace bytes echo_fp8_gemm needs for these sizes: 0 where it needs none
 * or the sizes are invalid (with a detail in echo_last_error() then).  They do not
 * fall with num_tokens: what the largest batch needs serves every smaller one.  At
 * most 256 MiB. */
size_t echo_fp8_gemm_workspace_bytes(int32_t num_tokens, int32_t out_features,
                                     int32_t in_features);

#ifdef __cplusplus
}
#endif

#endif /* ECHO_FP8_H */
