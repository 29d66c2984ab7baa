/*
 * comp_ams_operators.h - operators of language-model training next to the compressed optimiser of comp_ams.h:
 * layer norm, the softmax of attention scores with a learned relative position bias, log probabilities of tokens
 * with their alternatives, and distillation from a teacher's top logits - forward and, where a model trains
 * through them, backward.
 *
 * What they share with the optimiser is its data: parameters are fp32 and stand anywhere in the flat model theta;
 * gradients of parameters are reduced per worker and written straight into that worker's row of the gradient array
 * grads[n][d] that comp_ams_step takes (fp32, bfloat16 or half precision), so that one backward pass over the
 * microbatches of all workers replaces one pass per worker.
 *
 * Conventions
 *  - No handle.  Every call returns a status code of comp_ams.h, validates its arguments on the host before any
 *    device call, launches kernels on `hip_stream` (a hipStream_t of the current GPU, NULL = the null stream) and
 *    returns without waiting.  It allocates nothing, so it may be recorded into a HIP graph.  Of a call that is refused
 *    (COMP_AMS_EINVAL) nothing is launched; where a launch fails (COMP_AMS_EDEVICE) what depends on it is not launched, and
 *    outputs are undefined.  comp_ams_operators_last_error() describes the reason (per thread).
 *  - All pointers are device pointers of the current GPU unless they are named `host`.  Arrays of 16- and 32-bit
 *    elements need the alignment of their element only; strides are in elements and the last dimension is dense.
 *  - `type` is that of the activations (COMP_AMS_F32, COMP_AMS_BF16 or COMP_AMS_F16), `grad_type` that of the
 *    parameter gradients.  All arithmetic is fp32; sums, maxima, means and softmax statistics stay fp32, and a
 *    result is rounded once, to nearest even, when it is stored.
 *  - Results do not depend on timing: no sum is formed by atomics.
 *  - Unless said otherwise outputs must not overlap inputs or each other.
 */
#ifndef COMP_AMS_OPERATORS_H
#define COMP_AMS_OPERATORS_H

#include "comp_ams.h"

#ifdef __cplusplus
extern "C" {
#endif

enum { COMP_AMS_F32 = 0, COMP_AMS_BF16 = 1, COMP_AMS_F16 = 2 };

/* Most buckets of a relative position bias, and most tokens of a top list. */
enum { COMP_AMS_MAX_BUCKETS = 128, COMP_AMS_MAX_TOP = 128 };

/*
 * Layer norm of `rows` rows of `cols` elements:
 *   mean = (1/cols) sum x,  rstd = 1 / sqrt((1/cols) sum (x - mean)^2 + eps),  y = (x - mean) rstd gain + shift.
 * gain, shift: fp32 [cols]; shift may be NULL (no shift).  mean, rstd: fp32 [rows], kept for the backward pass; both
 * may be NULL.  The variance is taken from the differences.  rows >= 0, 1 <= cols < 2^31; y may be x itself with
 * the same stride.
 */
int comp_ams_layer_norm(void *y, float *mean, float *rstd, const void *x, const float *gain, const float *shift,
                        int64_t rows, int64_t cols, int64_t x_stride, int64_t y_stride, float eps, int32_t type,
                        void *hip_stream);

/*
 * Its backward pass.  With xh = (x - mean) rstd and a = dy gain:
 *   dx = rstd (a - (1/cols) sum a - xh (1/cols) sum a xh)           per row
 *   dgain[w] = sum dy xh,  dshift[w] = sum dy                        over the rows of worker w
 * Worker w of n (1 <= n <= 65535) holds the rows [w rows/n, (w + 1) rows/n); rows must be a multiple of n.  dgain and dshift point at
 * the parameter's place in worker 0's row; the next worker's is grad_stride elements further.  dshift may be NULL.
 * dx may be dy or x itself with the same stride.  With rows = 0 the parameter gradients are zero.
 * work: comp_ams_layer_norm_work_bytes() bytes of device memory, 16-byte aligned, not kept from one call to the next.
 */
int comp_ams_layer_norm_backward(void *dx, void *dgain, void *dshift, const void *dy, const void *x, const float *mean,
                                 const float *rstd, const float *gain, int64_t rows, int64_t cols, int64_t dx_stride,
                                 int64_t dy_stride, int64_t x_stride, int32_t n, int64_t grad_stride, int32_t type,
                                 int32_t grad_type, void *work, uint64_t work_bytes, void *hip_stream);
int comp_ams_layer_norm_work_bytes(int64_t rows, int64_t cols, int32_t n, uint64_t *bytes);

/*
 * Softmax of attention scores with a learned relative position bias, over [batch][heads][tq][tk] scores s:
 *   r = j - (i + offset)                                   position of key j relative to query i
 *   t_ij = scale s_ij + table[bucket(r)][head],            bucket(r) = how many of the bounds are <= r
 *   p_ij = exp(t_ij) / sum_j exp(t_ij)                     over the keys that query i sees, 0 elsewhere
 * A query sees key j if j < key_len[b] (key_len may be NULL: all) and, with causal != 0, if r <= 0.  What stands in the
 * score of a key that is not seen does not matter.  A query that sees nothing, or whose seen scores are all
 * -infinity, gets a row of zeros.  A NaN or a +infinity among the seen scores makes the row NaN.
 *   bounds_host: host memory, n_buckets - 1 strictly ascending relative positions (read before the call returns);
 *   1 <= n_buckets <= COMP_AMS_MAX_BUCKETS.  table: fp32 [n_buckets][heads].  key_len: int32 [batch], values outside
 *   [0, tk] count as the nearer end.
 * s_strides, p_strides: host arrays of three strides, {batch, head, query}.  batch, heads, tq, tk >= 0 with
 * tk < 2^31, tq < 2^30, batch heads tq < 2^31; |offset| < 2^31.  p may be s itself with the same strides.
 */
int comp_ams_rel_bias_softmax(void *p, const void *s, const float *table, const int32_t *bounds_host, int32_t n_buckets,
                              const int32_t *key_len, int64_t batch, int64_t heads, int64_t tq, int64_t tk,
                              const int64_t *p_strides_host, const int64_t *s_strides_host, int64_t offset, float scale,
                              int32_t causal, int32_t type, void *hip_stream);

/*
 * Its backward pass from the probabilities p and their gradient dp:
 *   dt_ij = p_ij (dp_ij - sum_j p_ij dp_ij),  ds = scale dt,  dtable[w][bucket][head] = sum of dt over worker w's
 *   sequences, its queries, and the keys in that bucket.
 * Worker w of n holds the sequences [w batch/n, (w + 1) batch/n); batch must be a multiple of n.  Keys that are not seen
 * (key_len, causal) and keys of probability zero take no gradient, whatever stands in dp there; ds is zero there.
 * dtable points at the table's place in worker 0's row, [n_buckets][heads] dense, the next worker's grad_stride further.
 * strides_host: nine strides, {batch, head, query} of ds, dp and p.  ds may be dp itself with the same strides.
 * work as above, comp_ams_rel_bias_work_bytes() bytes.
 */
int comp_ams_rel_bias_softmax_backward(void *ds, void *dtable, const void *dp, const void *p, const int32_t *bounds_host,
                                       int32_t n_buckets, const int32_t *key_len, int64_t batch, int64_t heads, int64_t tq,
                                       int64_t tk, const int64_t *strides_host, int64_t offset, float scale, int32_t causal,
                                       int32_t n, int64_t grad_stride, int32_t type, int32_t grad_type, void *work,
                                       uint64_t work_bytes, void *hip_stream);
int comp_ams_rel_bias_work_bytes(int64_t batch, int64_t heads, int64_t tq, int64_t tk, int32_t n_buckets, int32_t type, uint64_t *bytes);

/*
 * Log probabilities of given tokens under logits z of `rows` rows over a vocabulary, with the entropy of each
 * distribution and its k best tokens:
 *   lse = log sum_v exp(z_v),  logp = z_token - lse,  entropy = lse - sum_v p_v z_v,  p_v = exp(z_v - lse)
 *   top_idx[row][0..k-1]: the tokens of the k largest logits, largest first, the lower token first among equals
 *   (-0 equals +0; a NaN counts as larger than +infinity, NaNs among each other as equal), top_logp their log probabilities.
 * tokens: int64 [rows] or NULL (then logp is NULL too); a token outside [0, vocab) has logp = 0.  Any of logp,
 * entropy and, with k = 0, the top arrays may be NULL.  -infinity has probability zero; a row with a NaN, a +infinity or
 * nothing but -infinity has NaN for its log probabilities and entropy.  0 <= k <= min(vocab, COMP_AMS_MAX_TOP),
 * 1 <= vocab < 2^31.  work: comp_ams_token_logprobs_work_bytes() bytes, which may be 0 (then NULL will do).
 */
int comp_ams_token_logprobs(float *logp, float *entropy, int32_t *top_idx, float *top_logp, const void *logits,
                            const int64_t *tokens, int64_t rows, int64_t vocab, int64_t stride, int32_t k, int32_t type,
                            void *work, uint64_t work_bytes, void *hip_stream);
int comp_ams_token_logprobs_work_bytes(int64_t rows, int64_t vocab, int32_t k, int32_t type, uint64_t *bytes);

/*
 * Distillation from a teacher's top logits at a temperature T > 0.  The teacher's list of a row is idx[row][0..k-1]
 * (tokens; an entry outside [0, vocab) is not there) with val[row][0..k-1], its logits or log probabilities at
 * temperature 1 up to a constant:
 *   q_j = exp(val_j / T) / sum over the listed,   lp_v = z_v / T - lse,  lse = log sum_v exp(z_v / T)
 *   loss = T^2 sum_j q_j (log q_j - lp_{idx_j})
 * and, for a gradient dloss of the row's loss,
 *   dz_v = dloss T (exp(lp_v) - sum of q_j over the j with idx_j = v).
 * A row whose list is empty has loss 0 and gradient 0.  Entries with val = -infinity are listed with q = 0; if all are, the loss is 0 and
 * the gradient that of the probabilities alone.
 * idx: int32, val: fp32, dense [rows][k], 1 <= k <= COMP_AMS_MAX_TOP; 1 <= vocab < 2^31.
 *   comp_ams_distill           writes loss [rows] and lse [rows] (either may be NULL)
 *   comp_ams_distill_backward  writes dz [rows][vocab] from lse and dloss.  lse has been rounded to fp32, which the probabilities carry
 *                              (|lse| 2^-24, relative): logits of 10^4 cost them three digits, and of rows beyond 2^24 - masked throughout
 *                              with a large number - they are not known from it at all; comp_ams_distill_grad has no such limit
 *   comp_ams_distill_grad      both at once, for a loss whose weights (dloss) are known beforehand: one pass over the
 *                              logits; loss may be NULL
 * dlogits may be logits itself with the same stride.
 */
int comp_ams_distill(float *loss, float *lse, const void *logits, const int32_t *idx, const float *val, int64_t rows,
                     int64_t vocab, int64_t stride, int32_t k, float temperature, int32_t type, void *hip_stream);
int comp_ams_distill_backward(void *dlogits, const float *dloss, const void *logits, const float *lse, const int32_t *idx,
                              const float *val, int64_t rows, int64_t vocab, int64_t dlogits_stride, int64_t stride, int32_t k,
                              float temperature, int32_t type, void *hip_stream);
int comp_ams_distill_grad(float *loss, void *dlogits, const float *dloss, const void *logits, const int32_t *idx,
                          const float *val, int64_t rows, int64_t vocab, int64_t dlogits_stride, int64_t stride, int32_t k,
                          float temperature, int32_t type, void *hip_stream);

/* Message of the calling thread's last failure among the calls above. */
const char *comp_ams_operators_last_error(void);

#ifdef __cplusplus
}
#endif
#endif /* COMP_AMS_OPERATORS_H */
