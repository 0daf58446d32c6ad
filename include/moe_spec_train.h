/* Operators for training the expert estimator (paper: Sec. 6, Appendix A) and the routers it learns from, for one
 * AMD MI355X (gfx950).  Beside include/moe_spec.h, whose contexts run the trained estimator.
 *
 *   LayerNorm            y = (x - mean) * rstd * gain + bias over each row, and its backward pass with the sums over all
 *                        rows that are the gradients of gain and bias
 *   distillation loss    mean over the valid rows of KL(softmax(teacher / tau) || softmax(student / tau)), and its gradient
 *                        with respect to the student's logits
 *   balance loss         coef * E * sum_e f_e P_e with f_e = count_e / (n k) the share of the n valid rows' k choices that
 *                        expert e got and P_e the mean of softmax(logits)_e over the valid rows; the counts; and the
 *                        gradient with respect to the logits (the counts have none)
 *   AdamW                one step over many tensors, moments in 32 or in 8 bits
 *
 * Every call queues kernels on `stream` (a hipStream_t) and returns; it allocates nothing, waits for nothing and keeps no
 * state, so it can be captured into a HIP graph.  "dev" pointers are memory of the stream's device, which need not be the
 * current one (the null stream's is).  Tensors are row-major: the last dimension is contiguous, rows are `*_stride` elements apart.  An output's
 * stride is at least its row length; an input's may be anything from 0 (one row for all) on.  Pointers need the alignment of
 * their elements and no more.  Outputs must not overlap inputs, except where an in-place form is named.  The same inputs
 * give the same bits: no atomics on floating-point values.  Values are bfloat16 or float (MOE_SPEC_BF16, MOE_SPEC_F32);
 * statistics, sums and moments are held in float or wider, and what goes out as bfloat16 is rounded once, to nearest even.
 *
 * Calls that need scratch take a workspace (dev, 16-byte aligned) of at least the bytes that the matching function names (0 for
 * small sizes: NULL will do; also 0 for sizes that the call refuses).  Nothing in it has to be set and nothing is kept in it,
 * but two calls, or replays of two graphs, that may run at the same time need two.
 *
 * Returns 0 (MOE_SPEC_OK), MOE_SPEC_EINVAL for arguments it refuses (nothing has been queued then) or MOE_SPEC_EHIP;
 * moe_spec_train_last_error gives the reason of the calling thread's last failure.  Nothing throws or aborts. */
#ifndef MOE_SPEC_TRAIN_H
#define MOE_SPEC_TRAIN_H

#include <stddef.h>
#include <stdint.h>

#include "moe_spec.h"

#ifdef __cplusplus
extern "C" {
#endif

#define MOE_SPEC_TRAIN_MAX_COLS 8192          /* widest row of LayerNorm */
#define MOE_SPEC_TRAIN_MAX_ROWS 0x7fffffff
#define MOE_SPEC_TRAIN_MAX_TENSORS 65536      /* of one AdamW call */
#define MOE_SPEC_ADAMW_MAX_ELEMENTS 34359736320  /* of one of its tensors: what the threads of a launch, below 2^32, take */

/* LayerNorm (Appendix A: the estimator's last step before its head).  x, y dev [rows, cols]; gain, bias dev [cols] float or
 * NULL (ones, zeros); mean, rstd dev [rows] float or NULL: the row's mean and 1 / sqrt(variance + eps), which the backward
 * pass reads.  y may be x itself with the same stride. */
int moe_spec_layernorm_forward(void *stream, int dtype, const void *x, int64_t x_stride, int64_t rows, int cols,
                               const float *gain, const float *bias, float eps, void *y, int64_t y_stride, float *mean,
                               float *rstd);

/* Its backward pass.  dy, x dev [rows, cols]; mean, rstd as the forward pass left them; gain as there.
 * dx dev [rows, cols] or NULL; dgain, dbias dev [cols] float or NULL, written, not added to (zeros where rows = 0). */
size_t moe_spec_layernorm_backward_workspace_bytes(int64_t rows, int cols);
int moe_spec_layernorm_backward(void *stream, int dtype, const void *dy, int64_t dy_stride, const void *x, int64_t x_stride,
                                int64_t rows, int cols, const float *mean, const float *rstd, const float *gain, void *dx,
                                int64_t dx_stride, float *dgain, float *dbias, void *workspace, size_t workspace_bytes);

/* Distillation from a router (Appendix A: KL divergence from the true router's distribution).  student, teacher dev
 * [rows, n_experts], 1 <= n_experts <= MOE_SPEC_MAX_EXPERTS, each of a type of its own; temperature > 0 divides both.
 * valid dev [rows] bytes or NULL: rows whose byte is 0 (padding) count for nothing, whatever they hold; their gradients are
 * zero.  loss dev, one float: 0 if no row is valid.  grad dev [rows, n_experts] in the student's type or NULL; it may be
 * `student` itself with the same stride.
 * A logit of minus infinity has probability zero.  Where the teacher's is, nothing is added to the loss; a row whose
 * teacher has no other logits teaches nothing: loss and gradient zero (it counts in the mean).  Where only the student's is,
 * the loss is infinite, however small the teacher's probability, and the gradient finite; a difference between logits of a
 * row that float cannot hold counts as infinite.  Any other logit that is no finite number makes the loss and that row's
 * gradient NaN, and no other row's. */
size_t moe_spec_distill_loss_workspace_bytes(int64_t rows, int n_experts);
int moe_spec_distill_loss(void *stream, int student_dtype, const void *student, int64_t student_stride, int teacher_dtype,
                          const void *teacher, int64_t teacher_stride, int64_t rows, int n_experts, float temperature,
                          const uint8_t *valid, float *loss, void *grad, int64_t grad_stride, void *workspace,
                          size_t workspace_bytes);

/* Balance of a router's choices.  logits dev [rows, n_experts]; ids dev [rows, top_k] int32, 1 <= top_k <=
 * MOE_SPEC_MAX_TOP_K, as the layer steps report them (true_ids); an id outside [0, n_experts) is no choice and is not
 * counted, one that a row names twice counts twice.  valid, loss, grad as above; rows * top_k must be below 2^31.
 * counts dev [n_experts] int32.  A row of logits that are all minus infinity has no probabilities to give: gradient zero. */
size_t moe_spec_balance_loss_workspace_bytes(int64_t rows, int n_experts, int top_k);
int moe_spec_balance_loss(void *stream, int dtype, const void *logits, int64_t logits_stride, int64_t rows, int n_experts,
                          const int32_t *ids, int64_t ids_stride, int top_k, float coef, const uint8_t *valid, float *loss,
                          int32_t *counts, void *grad, int64_t grad_stride, void *workspace, size_t workspace_bytes);

/* AdamW.  With g = scale * grad and t the number of the step, counted from 1:
 *   m = beta1 m + (1 - beta1) g;  v = beta2 v + (1 - beta2) g^2
 *   p = p (1 - lr weight_decay) - lr / (1 - beta1^t) * m / (sqrt(v) / sqrt(1 - beta2^t) + eps)
 * in float, one rounding an operation.  The parameters are float; each tensor may name a bfloat16 copy, written rounded to
 * nearest even, as moe_spec_set_estimator and moe_spec_set_layer_resident read weights.
 *
 * Moments in 8 bits (MOE_SPEC_MOMENTS_8BIT).  Each run of 128 elements of a tensor has one byte for either moment: the
 * biased exponent X (the float format's) of the largest finite magnitude among them.  A first moment is a sign, four bits of
 * exponent and three of mantissa; a second moment, which has no sign, four and four: a value is
 * float_with_bits(code << 20 or code << 19) * 2^(X - 14).  The largest has exponent field 14; the last code (127 / 255) is
 * NaN and stands for infinities too.  A second moment that is not zero is never stored as zero.
 * Codes are rounded up or down at random, without bias, by 16 bits each from a mix of seed, t, the tensor's place in the
 * call and the lower 32 bits of the element's in the tensor.
 * To nearest would not do: with beta2 = 0.999 a step moves v by about a thousandth,
 * half a step of the code is 1.6 to 3 %, and v would stand still.  The price is noise: a step that moves v by d < h, h the
 * code's step, does so with variance d h, so at beta2 = 0.999 and normally distributed gradients v wanders about its 32-bit
 * value with a relative standard deviation of about 0.15 (0.07 for the square root, which divides); m with one of 0.09
 * at beta1 = 0.9.  p itself is updated from the unrounded moments of the step. */
enum { MOE_SPEC_MOMENTS_32BIT = 0, MOE_SPEC_MOMENTS_8BIT = 1 };
#define MOE_SPEC_MOMENT_BLOCK 128

typedef struct {
  float *p;                       /* dev [n], updated */
  const void *grad;               /* dev [n], in grad_dtype */
  void *m, *v;                    /* dev [n] float, or bytes with 8-bit moments; updated; zeros before the first step */
  uint8_t *m_exp, *v_exp;         /* dev [(n + 127) / 128], 8-bit moments only; updated; zeros before the first step */
  void *copy;                     /* dev [n] bfloat16, or NULL */
  int64_t n;
} moe_spec_adamw_tensor;

typedef struct {
  double lr, beta1, beta2, eps, weight_decay, grad_scale;
  int64_t step;                   /* t >= 1, unless step_dev is given */
  const int64_t *step_dev;        /* dev, or NULL: where the kernels read t (below 1: 1), for captured graphs; the caller
                                     advances it */
  const float *grad_scale_dev;    /* dev, or NULL: a second factor of the gradients (a clipping factor, a loss scale) */
  uint32_t seed;
  int32_t grad_dtype;             /* MOE_SPEC_F32 | MOE_SPEC_BF16 */
  int32_t moments;                /* MOE_SPEC_MOMENTS_* */
} moe_spec_adamw_config;

/* tensors: host [n_tensors], read before the call returns; no two of them may share memory that is updated. */
int moe_spec_adamw_step(void *stream, const moe_spec_adamw_tensor *tensors, int n_tensors, const moe_spec_adamw_config *cfg);

/* The values of 8-bit moments (p, grad and copy are not looked at): m_out[i], v_out[i] dev [n] in out_dtype (bfloat16 holds
 * all from 2^-120 on exactly), host arrays of n_tensors pointers; either array may be NULL. */
int moe_spec_adamw_read_moments(void *stream, const moe_spec_adamw_tensor *tensors, int n_tensors, int out_dtype,
                                void *const *m_out, void *const *v_out);

/* Text of the calling thread's last failure among the calls above. */
const char *moe_spec_train_last_error(void);

#ifdef __cplusplus
}
#endif
#endif /* MOE_SPEC_TRAIN_H */
