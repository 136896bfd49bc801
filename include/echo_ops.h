/*
 * echo_ops.h -- C ABI of the training-step operators of libecho.so.
 *
 * The composer (echo.h) plans training jobs from the durations of their operators.  These are the
 * operators that a pipeline stage of such a job runs outside its matrix products -- embedding lookup,
 * layer norm, cross entropy, and their gradients -- so that their durations, and what they compute,
 * can be had on the GPU at hand.
 *
 * Conventions, besides those of echo.h (return codes, echo_last_error, asynchronous work on the
 * caller's stream, nothing throws):
 *   - every pointer is device memory of GPU `hip_device` and belongs to the caller; the calling
 *     thread's current device is left as it was;
 *   - `type` is the element type of activations (ECHO_F32, ECHO_F16, ECHO_BF16); arithmetic, sums and
 *     softmax statistics are in 32 bits and each output is rounded once;
 *   - a matrix argument is `rows` rows of `cols` contiguous elements, `*_stride` elements apart
 *     (0 to 2^28; 0 repeats one row).  Elements need the alignment of their type only.  Outputs without a
 *     stride argument are dense.  0 <= rows < 2^31, 1 <= cols <= 2^24, and rows * cols <= 2^38 (else
 *     ECHO_ERR_RANGE);
 *   - outputs may not overlap inputs or each other unless a call says so (ECHO_ERR_ARG).  Rows of one stride may lie
 *     between each other's, as the column halves of one buffer do;
 *   - workspaces are scratch: their contents need no initialisation and mean nothing after the call,
 *     so calls on one stream may share one.  Nothing is allocated, cleared by memset or waited for, so
 *     every call can be recorded by HIP stream capture;
 *   - results do not depend on the run: sums are taken in an order that the sizes fix.
 */
#ifndef ECHO_OPS_H
#define ECHO_OPS_H

#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

enum { ECHO_F32 = 0, ECHO_F16 = 1, ECHO_BF16 = 2 };   /* element types          */
enum { ECHO_I32 = 0, ECHO_I64 = 1 };                  /* token ids and targets  */

/*
 * Layer norm over the last dimension, with the residual add in front of it.
 *   h = x + residual, rounded to `type` (residual NULL: h = x)
 *   mean = sum h / cols,  rstd = 1 / sqrt(sum (h - mean)^2 / cols + eps)
 *   y = (h - mean) * rstd * weight + bias
 * weight and bias (may be NULL: 0) hold cols elements of weight_type, which is `type` or ECHO_F32.
 * y [rows][cols] of `type`; mean, rstd [rows] of 32 bits; sum [rows][cols] of `type` receives h and is
 * given exactly when residual is (it may be x or residual itself, where that is dense).
 * eps is finite and >= 0.
 */
int echo_layer_norm(const void *x, int64_t x_stride, const void *residual, int64_t residual_stride,
                    const void *weight, const void *bias, int32_t type, int32_t weight_type, int64_t rows,
                    int64_t cols, float eps, void *y, void *sum, float *mean, float *rstd, int hip_device,
                    void *hip_stream);

/*
 * Gradients of echo_layer_norm from that of y.  x is the normalised input (h), mean and rstd its saved
 * statistics; with n = (x - mean) * rstd and g = dy * weight:
 *   dx = rstd * (g - mean(g) - n * mean(g * n)) + grad_residual
 *   dweight = sum over rows of dy * n,   dbias = sum over rows of dy
 * grad_residual (NULL: 0) is the gradient that reaches h past the norm.  dx [rows][cols] of `type` (it may
 * be dy or grad_residual itself, where that is dense).  dweight, dbias (dbias may be NULL) hold cols elements
 * of grad_type (weight_type or ECHO_F32) and are written, or with accumulate != 0 added to.
 * workspace: at least echo_layer_norm_grad_workspace(rows, cols) bytes, aligned to 16.
 */
int64_t echo_layer_norm_grad_workspace(int64_t rows, int64_t cols);
int echo_layer_norm_grad(const void *dy, int64_t dy_stride, const void *x, int64_t x_stride, const void *weight,
                         const float *mean, const float *rstd, const void *grad_residual,
                         int64_t grad_residual_stride, int32_t type, int32_t weight_type, int64_t rows, int64_t cols,
                         void *dx, void *dweight, void *dbias, int32_t grad_type, int32_t accumulate,
                         void *workspace, int64_t workspace_bytes, int hip_device, void *hip_stream);

/*
 * Embedding lookup in the rows [vocab_start, vocab_start + vocab) of a table:
 *   out[t] = scale * weight[ids[t] - vocab_start], or a row of zeros where that row is not held here
 * (another rank's, or no id at all: any value is allowed in ids).  ids [rows], weight [vocab] rows of cols
 * elements, out [rows][cols], weight and out of `type`.  0 <= vocab < 2^31.
 */
int echo_embedding(const void *ids, int32_t index_type, const void *weight, int64_t weight_stride, int32_t type,
                   int64_t rows, int64_t cols, int64_t vocab_start, int64_t vocab, float scale, void *out,
                   int hip_device, void *hip_stream);

/*
 * Gradient of echo_embedding's table:
 *   dweight[v] = scale * sum of dy[t] over the t with ids[t] = vocab_start + v
 * for every row of the shard (zeros where no token has the id), or with accumulate != 0 added to
 * dweight, whose other rows are then left alone.  dy is of `type`, dweight [vocab][cols] of grad_type
 * (`type` or ECHO_F32); vocab <= 2^26, rows <= 2^29 and rows * vocab <= 2^42 (else ECHO_ERR_RANGE).  Tokens are
 * sorted by id first, by vocab / 64 workgroups that each look through all of them; a row's tokens are summed in
 * chunks of ascending order, and the chunks joined in an order that the sizes fix.
 * workspace: at least echo_embedding_grad_workspace(rows, cols, vocab) bytes, aligned to 16.
 */
int64_t echo_embedding_grad_workspace(int64_t rows, int64_t cols, int64_t vocab);
int echo_embedding_grad(const void *ids, int32_t index_type, const void *dy, int64_t dy_stride, int32_t type,
                        int64_t rows, int64_t cols, int64_t vocab_start, int64_t vocab, float scale, void *dweight,
                        int32_t grad_type, int32_t accumulate, void *workspace, int64_t workspace_bytes,
                        int hip_device, void *hip_stream);

/*
 * Cross entropy of rows of logits over the ids [vocab_start, vocab_start + cols) of a vocabulary of
 * vocab_size ids (the others belong to other ranks).  A row whose target lies outside [0, vocab_size) is
 * not trained on.  Per row (any of lse, target, loss may be NULL; 32 bits):
 *   lse     log of the sum of exp(logits): -inf where every logit is -inf, NaN where the row has a NaN or +inf
 *   target  the target's logit; 0 where it is not held here or the row is not trained on
 *   loss    lse - target, before lse is rounded; 0 for a row not trained on, +inf where the target's logit is -inf,
 *           NaN where the row has a NaN or +inf (whole vocabulary only)
 *   grad    (exp(logit - lse) - [v = target]) * grad_loss[row], [rows][cols] of `type` (whole vocabulary
 *           only): the gradient, in the same pass, for a grad_loss [rows] known beforehand.  Rows not
 *           trained on and rows without a finite logit get zeros.  May be logits itself.
 * For a vocabulary over several ranks, the whole lse is log(sum over ranks of exp(lse)), the target's
 * logit the sum over ranks, and echo_cross_entropy_grad gives each rank its gradient.
 */
int echo_cross_entropy(const void *logits, int64_t logits_stride, int32_t type, const void *targets,
                       int32_t index_type, int64_t rows, int64_t cols, int64_t vocab_start, int64_t vocab_size,
                       float *lse, float *target, float *loss, const float *grad_loss, void *grad,
                       int64_t grad_stride, int hip_device, void *hip_stream);

/*
 * grad = (exp(logits - lse) - [v = target]) * grad_loss for the columns held here, lse [rows] that of
 * the whole vocabulary.  Rows not trained on and rows with lse = -inf get zeros.  grad may be logits itself.
 * lse is taken as it is given: in a row masked throughout with a value so low that the logarithm is below lse's last place,
 * the probabilities are those of that rounded lse (echo_cross_entropy's own gradient has the maximum and the sum).
 */
int echo_cross_entropy_grad(const void *logits, int64_t logits_stride, int32_t type, const void *targets,
                            int32_t index_type, int64_t rows, int64_t cols, int64_t vocab_start, int64_t vocab_size,
                            const float *lse, const float *grad_loss, void *grad, int64_t grad_stride,
                            int hip_device, void *hip_stream);

#ifdef __cplusplus
}
#endif

#endif /* ECHO_OPS_H */
