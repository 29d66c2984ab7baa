/*
 * comp_ams_rows8.h - operators of language-model training and serving on rows held in 8 bits, next to those of
 * comp_ams_operators.h: the root-mean-square norm with the residual's addition and an output in 8 bits, activation checkpoints
 * in 8 bits, the weight gradients of a linear layer formed from them per worker, and the product of 8-bit integers with a
 * scale for each token and channel.
 *
 * A row in 8 bits is q[cols] (int8) and one fp32 scale:
 *   scale = max(absmax / 127, 2^-126), with binary != 0 the least power of two not below that,  q = rint(x (1 / scale))
 * in fp32, every operation rounded on its own, rint to even.  |q| is at most 127, and less where 127 scale would leave the type that the
 * row came from.  It stands for q scale.  A row with a NaN or an infinity has the scale NaN and zeros in q.  Scales that are powers of two make q scale exact
 * in fp32, bfloat16 and half precision (where it is in range) and cost half a bit on average.
 *
 * Conventions are those of comp_ams_operators.h (status codes, streams, alignment, types, no allocation, graphs, errors through
 * comp_ams_operators_last_error()); arrays of int8 may stand at any byte.
 */
#ifndef COMP_AMS_ROWS8_H
#define COMP_AMS_ROWS8_H

#include "comp_ams_operators.h"

#ifdef __cplusplus
extern "C" {
#endif

/* One more than the largest number of input channels of comp_ams_linear_q8: sums of 2^17 products of 8 bits may leave 32 bits. */
enum { COMP_AMS_MAX_Q8_COLS = 131072 };

/*
 * x [rows][cols] to 8 bits, and back:  q, scale from x;  x = q scale, rounded once.  rows, cols >= 0; rows < 2^31, cols < 2^31.
 * q: int8 rows `q_stride` apart; scale: fp32 [rows].  `type` is that of x.
 */
int comp_ams_quantize_rows(int8_t *q, float *scale, const void *x, int64_t rows, int64_t cols, int64_t q_stride, int64_t x_stride,
                           int32_t binary, int32_t type, void *hip_stream);
int comp_ams_restore_rows(void *x, const int8_t *q, const float *scale, int64_t rows, int64_t cols, int64_t x_stride, int64_t q_stride,
                          int32_t type, void *hip_stream);

/*
 * Root-mean-square norm of `rows` rows of `cols` elements, after the residual's addition:
 *   h = x + residual, rounded to the type;  rstd = 1 / sqrt((1/cols) sum h^2 + eps);  y = (h rstd) gain
 * residual may be NULL (h = x).  h (the residual stream that the next layer and the backward pass read) may be NULL: not stored;
 * rstd: fp32 [rows], may be NULL.  gain: fp32 [cols].  The squares are summed in fp32: a row whose sum leaves it has rstd = 0.
 * 0 <= rows < 2^40, 1 <= cols < 2^31.  h or y may be x or residual itself with the same stride, not both the same array.
 * comp_ams_rms_norm_q8 writes y in 8 bits (the scale from the fp32 values of y), for a product in 8 bits and as the checkpoint that
 * the product's weight gradient reads.
 */
int comp_ams_rms_norm(void *y, void *h, float *rstd, const void *x, const void *residual, const float *gain, int64_t rows, int64_t cols,
                      int64_t y_stride, int64_t h_stride, int64_t x_stride, int64_t residual_stride, float eps, int32_t type,
                      void *hip_stream);
int comp_ams_rms_norm_q8(int8_t *q, float *scale, void *h, float *rstd, const void *x, const void *residual, const float *gain,
                         int64_t rows, int64_t cols, int64_t q_stride, int64_t h_stride, int64_t x_stride, int64_t residual_stride,
                         float eps, int32_t binary, int32_t type, void *hip_stream);

/*
 * Its backward pass.  With xh = h rstd and a = dy gain:
 *   dx = rstd (a - xh (1/cols) sum a xh) + dresidual             per row: the gradient of x and of residual alike
 *   dgain[w] = sum dy xh                                          over the rows of worker w
 * h in the type of dy, or, with h_scale not NULL, int8 with a scale for each row (a checkpoint by comp_ams_quantize_rows).
 * dresidual: the gradient that reaches h past the norm, may be NULL.  Workers, gradients and work memory
 * (comp_ams_rms_norm_work_bytes()) as for comp_ams_layer_norm_backward.  dx may be dy, dresidual or an h of its type itself with the
 * same stride.  With rows = 0 the gradients are zero.
 */
int comp_ams_rms_norm_backward(void *dx, void *dgain, const void *dy, const void *h, const float *h_scale, const float *rstd,
                               const float *gain, const void *dresidual, int64_t rows, int64_t cols, int64_t dx_stride,
                               int64_t dy_stride, int64_t h_stride, int64_t dresidual_stride, int32_t n, int64_t grad_stride,
                               int32_t type, int32_t grad_type, void *work, uint64_t work_bytes, void *hip_stream);
int comp_ams_rms_norm_work_bytes(int64_t rows, int64_t cols, int32_t n, uint64_t *bytes);

/*
 * Product of 8-bit integers with a scale for each token and channel:
 *   y[r][o] = (sum_i q[r][i] w[o][i]) scale[r] w_scale[o] + bias[o]
 * q: int8 [rows][cols], w: int8 [outs][cols] (any values, -128 too), bias: fp32 [outs] or NULL.  The sum is exact, scales and bias are
 * applied in fp32 from left to right, y is rounded once to `type`.  0 <= rows, outs < 2^31, 0 <= cols < COMP_AMS_MAX_Q8_COLS.
 * With cols = 0 y is the bias.  The input's gradient is another such product: of dy in 8 bits with the transposed weight in 8 bits.
 * work: comp_ams_linear_q8_work_bytes() bytes of device memory, 16-byte aligned, which may be 0 (then NULL will do); fewer where, as q_aligned
 * and w_aligned != 0 promise, the array's address and stride are multiples of 16 and its stride is below 2^22.  (Rows are then read where
 * they stand, if cols is a multiple of 16 too.  Few rows need no work memory; how many depends on the sizes.)
 */
int comp_ams_linear_q8(void *y, const int8_t *q, const float *scale, const int8_t *w, const float *w_scale, const float *bias,
                       int64_t rows, int64_t cols, int64_t outs, int64_t y_stride, int64_t q_stride, int64_t w_stride, int32_t type,
                       void *work, uint64_t work_bytes, void *hip_stream);
int comp_ams_linear_q8_work_bytes(int64_t rows, int64_t cols, int64_t outs, int32_t q_aligned, int32_t w_aligned, uint64_t *bytes);

/*
 * Weight gradients of a linear layer y = x W^T + bias from its input in 8 bits, per worker:
 *   dweight[w][o][i] = sum dy[r][o] q[r][i] scale[r],  dbias[w][o] = sum dy[r][o]        over the rows r of worker w
 * Workers as for comp_ams_layer_norm_backward.  dweight points at the weight's place in worker 0's row, dense, [outs][cols], or [cols][outs]
 * with in_first != 0; dbias (may be NULL) at the bias'; the next worker's are grad_stride elements further.
 * Sums are fp32.  Before the product dy[r][o] scale[r] is rounded to fp32 and then, for dy and gradients in 16 bits, to 16 bits of mantissa; of bfloat16 it may
 * be q[r][i] scale[r] in its place.  binary != 0 promises that all scales are powers of two, as binary quantising gives them: of dy in 16 bits nothing is
 * lost then (but of numbers below 2^-126), and bfloat16 takes one product, half precision two, in place of two or, for fp32 gradients, three.
 * Where the promise does not hold, q scale is rounded to bfloat16, of half precision dy scale to 16 bits of mantissa.
 * An infinity or a NaN in dy or a scale reaches the worker's gradients that it belongs to, as an infinity or a NaN.
 * rows >= 0 a multiple of n and below 2^32, a worker's below 2^29; 0 <= cols, outs <= 2^23.  With rows = 0 the gradients are zero.
 * work: comp_ams_linear_weight_grad_work_bytes() bytes, 16-byte aligned, not kept from one call to the next: q in 16 bits, and dy too
 * unless one product takes it, outs is a multiple of 8 and, as dy_aligned != 0 promises, dy and its stride are multiples of 16 bytes; enough for
 * gradients of either width.
 */
int comp_ams_linear_weight_grad(void *dweight, void *dbias, const void *dy, const int8_t *q, const float *scale, int64_t rows,
                                int64_t cols, int64_t outs, int64_t dy_stride, int64_t q_stride, int32_t n, int64_t grad_stride,
                                int32_t in_first, int32_t binary, int32_t type, int32_t grad_type, void *work, uint64_t work_bytes,
                                void *hip_stream);
int comp_ams_linear_weight_grad_work_bytes(int64_t rows, int64_t cols, int64_t outs, int32_t n, int32_t binary, int32_t type,
                                           int32_t dy_aligned, uint64_t *bytes);

#ifdef __cplusplus
}
#endif
#endif /* COMP_AMS_ROWS8_H */
