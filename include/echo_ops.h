/*
 * echo_ops.h -- C ABI of the training-step operators of libecho.so.
 *
 * The composer (echo.h) plans training jobs from the durations of their operators.  These are the
 * operators that a pipeline stage of such a job runs outside its layers' matrix products -- embedding lookup,
 * layer norm, cross entropy, distillation, the output head with either loss, and their gradients -- so that
 * their durations, and what they compute, can be had on the GPU at hand.
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

/*
 * Distillation of rows of logits over the ids [vocab_start, vocab_start + cols) of a vocabulary of vocab_size ids from a
 * teacher's top logits: `top` ids a row and their logits, ids [rows][top] and teacher [rows][top] of teacher_type (`type` or
 * ECHO_F32), 1 <= top <= 1024.  Ids outside [0, vocab_size) are padding.  With T the temperature (1e-6 to 1e6), q the softmax of
 * teacher / T over the row's entries whose ids are in the vocabulary, one q an entry, and p that of logits / T over the
 * vocabulary, per row (any of lse, target, entropy, loss may be NULL; 32 bits):
 *   lse      log of the sum of exp(logits / T): -inf where every logit is -inf, NaN where the row has a NaN or +inf
 *   target   sum of q * logit / T over the entries whose ids are held here
 *   entropy  -sum of q log q over all entries of the row
 *   loss     T^2 * sum over the entries of q (log q - log p of its id); 0 for a row without an id whose logit is above -inf, which
 *            is not trained on, +inf where q is not 0 and the logit is -inf (whole vocabulary only)
 *   grad     T (p - q) * grad_loss[row], [rows][cols] of `type` (whole vocabulary only), in the same pass.  Rows not
 *            trained on and rows without a finite logit get zeros.  May be logits itself.
 * Where a row's ids are all different, loss is T^2 times the divergence of p from q.  An id may come more than once: in grad and
 * target its entries' q add up, while entropy and loss stay sums over the entries, each with its own log q.  Two entries q1 and q2
 * of one id have a loss below that of one entry q1 + q2, by T^2 ((q1 + q2) log(q1 + q2) - q1 log q1 - q2 log q2), a
 * constant of the student; the loss of such a row may be below 0.  Who wants the divergence there gives one entry an id, of
 * logit T log(sum of exp(teacher / T) over its entries).
 * For a vocabulary over several ranks, every rank is given all of a row's ids; the whole lse is log(sum over ranks of
 * exp(lse)), loss = T^2 * (lse - sum over ranks of target - entropy), and echo_distillation_grad gives each rank its gradient.
 */
int echo_distillation(const void *logits, int64_t logits_stride, int32_t type, const void *ids, int32_t index_type,
                      const void *teacher, int32_t teacher_type, int64_t rows, int64_t cols, int64_t top,
                      int64_t vocab_start, int64_t vocab_size, float temperature, float *lse, float *target,
                      float *entropy, float *loss, const float *grad_loss, void *grad, int64_t grad_stride,
                      int hip_device, void *hip_stream);

/*
 * grad = T (exp(logits / T - lse) - q) * grad_loss for the columns held here, logits / T as numbers of 32 bits and lse [rows]
 * that of the whole vocabulary, taken as it is given.  Rows not trained on and rows with lse = -inf get zeros.  grad may be logits itself.
 */
int echo_distillation_grad(const void *logits, int64_t logits_stride, int32_t type, const void *ids, int32_t index_type,
                           const void *teacher, int32_t teacher_type, int64_t rows, int64_t cols, int64_t top,
                           int64_t vocab_start, int64_t vocab_size, float temperature, const float *lse,
                           const float *grad_loss, void *grad, int64_t grad_stride, int hip_device, void *hip_stream);

/*
 * The same losses straight from hidden states [rows][cols] and an output table, `vocab` rows of cols elements for the ids
 * [vocab_start, vocab_start + vocab): logits = hidden weight^T, which are not returned.  hidden and weight are of `type`; the
 * products are of 16-bit elements (three of them for one of 32 bits) with sums in 32 bits, and logits, statistics and losses
 * are in 32 bits.  Gradients (both or neither), of the loss sum over rows of grad_loss * loss, with d the logits'
 * gradient of above:
 *   dhidden = d weight, [rows][cols] of `type`;   dweight = d^T hidden, [vocab][cols] of grad_type (`type` or ECHO_F32),
 *   written, or with accumulate != 0 added to.
 * Of 16-bit types d is rounded to `type` (relative to the largest finite |grad_loss| of the rows trained on) before these
 * products, as the logits' gradient of echo_cross_entropy is (of up to 64 rows it may be held in twice the bits); of 32 bits it
 * is held in 24.  Rows not trained on have d = 0.  A row whose hidden state has a NaN or an infinity gives NaN to every row of
 * dweight, trained on or not.  Logits / T beyond the largest number of 32 bits make lse infinite, and 32-bit elements beyond the
 * largest of bfloat16, infinities among them, count as NaN.
 * echo_linear_cross_entropy gives loss and gradients with the whole vocabulary (gradients together with lse), or a shard's lse
 * and target; echo_linear_cross_entropy_grad is given the whole vocabulary's lse: of ECHO_F16 one that is more than 1.38 below a
 * logit / T may overflow the gradients.  The distillations are their counterparts.
 * rows, vocab <= 2^24, cols <= 2^20, and the product of any two <= 2^38 (else ECHO_ERR_RANGE).
 * workspace: at least echo_linear_workspace(...) bytes for the same matrices, aligned to 16; top is 0 for the cross entropies,
 * loss and grads say which of the two the call computes.  It holds at most about 1 GiB of the logits' gradient at a time (256 columns
 * where those are more; once more in 32 bits for losses and gradients in one call of ECHO_F32 and ECHO_F16), besides
 * 32-bit sums of dhidden, statistics, and copies of matrices that the products do not take as they are: those of 32 bits, and those whose cols
 * are no multiple of 64, whose rows do not begin at multiples of 16 bytes or whose stride passes 2^22.
 */
int64_t echo_linear_workspace(const void *hidden, int64_t hidden_stride, const void *weight, int64_t weight_stride,
                              int32_t type, int64_t rows, int64_t cols, int64_t vocab, int64_t top, int32_t loss,
                              int32_t grads);
int echo_linear_cross_entropy(const void *hidden, int64_t hidden_stride, const void *weight, int64_t weight_stride,
                              int32_t type, const void *targets, int32_t index_type, int64_t rows, int64_t cols,
                              int64_t vocab, int64_t vocab_start, int64_t vocab_size, float *lse, float *target,
                              float *loss, const float *grad_loss, void *dhidden, void *dweight, int32_t grad_type,
                              int32_t accumulate, void *workspace, int64_t workspace_bytes, int hip_device,
                              void *hip_stream);
int echo_linear_cross_entropy_grad(const void *hidden, int64_t hidden_stride, const void *weight, int64_t weight_stride,
                                   int32_t type, const void *targets, int32_t index_type, int64_t rows, int64_t cols,
                                   int64_t vocab, int64_t vocab_start, int64_t vocab_size, const float *lse,
                                   const float *grad_loss, void *dhidden, void *dweight, int32_t grad_type,
                                   int32_t accumulate, void *workspace, int64_t workspace_bytes, int hip_device,
                                   void *hip_stream);
int echo_linear_distillation(const void *hidden, int64_t hidden_stride, const void *weight, int64_t weight_stride,
                             int32_t type, const void *ids, int32_t index_type, const void *teacher,
                             int32_t teacher_type, int64_t rows, int64_t cols, int64_t vocab, int64_t top,
                             int64_t vocab_start, int64_t vocab_size, float temperature, float *lse, float *target,
                             float *entropy, float *loss, const float *grad_loss, void *dhidden, void *dweight,
                             int32_t grad_type, int32_t accumulate, void *workspace, int64_t workspace_bytes,
                             int hip_device, void *hip_stream);
int echo_linear_distillation_grad(const void *hidden, int64_t hidden_stride, const void *weight, int64_t weight_stride,
                                  int32_t type, const void *ids, int32_t index_type, const void *teacher,
                                  int32_t teacher_type, int64_t rows, int64_t cols, int64_t vocab, int64_t top,
                                  int64_t vocab_start, int64_t vocab_size, float temperature, const float *lse,
                                  const float *grad_loss, void *dhidden, void *dweight, int32_t grad_type,
                                  int32_t accumulate, void *workspace, int64_t workspace_bytes, int hip_device,
                                  void *hip_stream);

#ifdef __cplusplus
}
#endif

#endif /* ECHO_OPS_H */
