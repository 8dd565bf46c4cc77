/*
 * ditint8.h -- linear layers in 8-bit integers, in libditstep.so and under the conventions of ditstep.h: the rollout's products
 * at twice the matrix rate and half the weight bytes of bf16. Weights are rounded once after an update, with a scale for each
 * output channel; activations are rounded in every call, with a scale for each token.
 *
 *   quantize_rows  rows to 8-bit integers with a scale each (weights [out][in]: a scale for each channel)
 *   int8_matmul    y = act(x W^T + b) of rows that are integers already
 *   int8_linear    the same of bf16 or fp32 rows, which it rounds first
 *
 * Every result is the same from run to run and does not depend on how a product is split: integer sums are exact.
 */
#ifndef DITINT8_H
#define DITINT8_H

#include <stddef.h>
#include <stdint.h>

#include "ditstep.h"

#ifdef __cplusplus
extern "C" {
#endif

/* For every row i of x [rows][cols] (dtype, row stride x_row elements):
 *   scale[i] = max(fp32(max_j |x[i][j]| / 127), 2^-126)
 *   q[i][j]  = the integer nearest to x[i][j] / scale[i], of two as near the even one (the quotient itself is rounded, not an
 *              fp32 quotient), in -127..127
 *   values[i][j] = q[i][j] scale[i], rounded to dtype: what the integers stand for (an update that follows an 8-bit
 *              rollout runs its own products with these; 127 scale may round past the largest fp32 number, to infinity, where
 *              max |x| is the largest)
 * A row that holds a NaN or an infinity gets scale NaN, q 0 and values NaN. q is int8 at row stride q_row; values (may be
 * NULL, may be x itself at its stride) has row stride values_row. Strides are at least cols; elements past cols are left as
 * they were. Tensors need the alignment of their type only. rows == 0 or cols == 0: no-op. */
dit_status quantize_rows(const void* x, int32_t rows, int32_t cols, int64_t x_row, int32_t dtype, int8_t* q, int64_t q_row,
                         float* scale, void* values, int64_t values_row, dit_stream stream);

typedef enum { DIT_ACT_NONE = 0, DIT_ACT_GELU_TANH = 1 } dit_activation;

typedef struct {
  int32_t rows;          /* of x and y, >= 0; y has at most 2^23 - 8 tiles of 256 x 256 results (2^39 of them) */
  int32_t in_features;   /* 1 .. 131071: the sums fit 32 bits whatever the integers are */
  int32_t out_features;  /* >= 0 */
  int32_t dtype;         /* dit_dtype of y and bias, and of int8_linear's x */
  int32_t act;           /* dit_activation */
  int64_t x_row;         /* row strides in elements: x (int8_matmul: a multiple of 16, at least in_features), */
  int64_t w_row;         /* w (a multiple of 16, at least in_features, below 2^23), */
  int64_t y_row;         /* y (at least out_features) */
} dit_int8_config;

/* Workspace bytes of the two calls (0 where none is needed, and for an invalid config). */
size_t int8_matmul_workspace_bytes(const dit_int8_config* cfg);
size_t int8_linear_workspace_bytes(const dit_int8_config* cfg);

/* y[i][n] = act( (sum_k x[i][k] w[n][k]) x_scale[i] w_scale[n] + bias[n] ). The sum is an exact integer; it is rounded to
 * fp32 and multiplied by x_scale, then by w_scale (so |sum x_scale| has to stay in the range of fp32), then the bias is added
 * and gelu_tanh taken, all in fp32 with one rounding to dtype at the end.
 *   x [rows][in] int8 at x_row, w [out][in] int8 at w_row: 16-byte aligned; what lies between in_features and the next
 *   multiple of 16 is read and does not count, so a row's storage goes that far
 *   x_scale [rows], w_scale [out] fp32; bias [out] (dtype) or NULL; y [rows][out] (dtype) at y_row
 * A NaN scale makes its row or channel of y NaN. rows == 0 or out_features == 0: no-op. */
dit_status int8_matmul(const dit_int8_config* cfg, const int8_t* x, const float* x_scale, const int8_t* w,
                       const float* w_scale, const void* bias, void* y, void* workspace, size_t workspace_bytes,
                       dit_stream stream);

/* int8_matmul of quantize_rows(x), x [rows][in] of dtype at x_row: the same result, bit for bit. y may not overlap x. */
dit_status int8_linear(const dit_int8_config* cfg, const void* x, const int8_t* w, const float* w_scale, const void* bias,
                       void* y, void* workspace, size_t workspace_bytes, dit_stream stream);

#ifdef __cplusplus
}
#endif
#endif /* DITINT8_H */
