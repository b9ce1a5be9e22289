/*
 * echo_int8.h -- linear layers in 8-bit integers (GPU).
 *
 * The decoder layer's products on operands held as signed 8-bit codes with one
 * fp32 scale per row: per token for activations [T][K], per output channel for
 * weights [N][K] (out_features x in_features).  The value of a code is
 * code * scale of its row.
 *
 * The conventions of echo.h hold: device pointers on the current device, work
 * enqueued on `stream`, nothing allocated, nothing kept, every check before
 * anything is enqueued, status codes with a detail in echo_last_error().
 * Tensors are row-major; strides are in elements.  A call of no rows returns
 * ECHO_OK and touches nothing (its pointers may be NULL).  Types are those of
 * echo_dtype_t (echo_fp8.h).
 */
#ifndef ECHO_INT8_H
#define ECHO_INT8_H

#include <stddef.h>
#include <stdint.h>

#include "echo_fp8.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Codes and scales of the rows of x [rows][cols] (bf16 or fp32, rows x_stride
 * elements apart):
 *   scale = fp32(amax / 127) over the row, 1 where that is 0;
 *   code  = the correctly rounded fp32 quotient x / scale, rounded to the nearest
 *           integer (ties to even), within +-127.
 * A row with a NaN or an infinity has the scale NaN and codes of 0, so that all
 * that is computed from it is NaN.
 * codes: [rows][cols]; scales: [rows].  cols a multiple of 16, at most 2^30; x and codes
 * 16-byte aligned, and x_stride >= cols with rows at 16-byte steps.  The buffers do not
 * overlap. */
int echo_int8_quantize(const void *x, int32_t x_dtype, int64_t x_stride, int32_t rows,
                       int32_t cols, int8_t *codes, float *scales, void *stream);

/* y[t][n] = x_scale[t] * w_scale[n] * sum_k x[t][k] w[n][k]  (+ bias[n]) (+ residual[t][n]),
 * x codes [T][K], w codes [N][K], any of -128 .. 127.  The sum is exact; it is
 * converted to fp32, scaled (no step of that leaves fp32's range where the scaled
 * sum does not), bias and residual are added in fp32 in this order, and y
 * [T][N], bf16 or fp32 with rows y_stride >= N elements apart, is rounded once.
 * Results do not hang on how a product is cut: a token's are the same in any batch.
 * bias (optional): fp32.  residual (optional): of y's type and strides; it may be y
 * itself, and overlaps it in no other way; y overlaps no other buffer.
 * K a multiple of 16, at most 131056 (sums of 32 bits); x and w 16-byte aligned.
 * workspace: device scratch of echo_int8_gemm_workspace_bytes() bytes (may be
 * none), 256-byte aligned, used by no other call until this one has completed. */
int echo_int8_gemm(const int8_t *x, const float *x_scale, const int8_t *w, const float *w_scale,
                   int32_t num_tokens, int32_t out_features, int32_t in_features,
                   const float *bias, const void *residual, void *y, int32_t y_dtype,
                   int64_t y_stride, void *workspace, size_t workspace_bytes, void *stream);

/* Workspace bytes echo_int8_gemm needs for these sizes: 0 where it needs none
 * or the sizes are invalid (with a detail in echo_last_error() then).  They do not
 * fall with num_tokens: what the largest batch needs serves every smaller one.  At
 * most 256 MiB. */
size_t echo_int8_gemm_workspace_bytes(int32_t num_tokens, int32_t out_features,
                                      int32_t in_features);

#ifdef __cplusplus
}
#endif

#endif /* ECHO_INT8_H */
