/* hh_train.h -- C ABI of what ends a training step on the last pipeline stage: the loss of the output projection with its
 * gradients, the global gradient norm with clipping, and the optimizer's update.
 *
 * The last stage of a pipeline (paper Section 2.3) turns its layers' output into a loss before its backward pass can begin,
 * and every device ends its step by clipping and applying the gradients that hh_layer_bwd has summed over the micro-batches:
 *
 *     hh_layer_fwd ... -> hh_head_step -> hh_layer_bwd ...   (each micro-batch)   -> hh_grad_clip -> hh_adamw_step
 *
 * The general rules of hh.h hold: statuses and hh_last_error(), device pointers, buffers that the caller owns, work enqueued on
 * `stream` without synchronisation, allocation or copies, checks of arguments before any of it.  Every result is the same
 * from run to run, bit for bit: no sum depends on the order in which workgroups finish.
 */
#ifndef HH_TRAIN_H
#define HH_TRAIN_H

#include "hh.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Output projection and softmax cross entropy.  With z = x W^T [T, V]:
 *     loss_t = log(sum_v exp z_tv) - z_t,label(t)
 *     step:  d_tv = g_t (exp(z_tv) / sum_u exp z_tu - [v = label(t)]),  g_t = scale * dloss_t (scale alone where dloss is NULL)
 *            dx = d W,   dW (+)= d^T x
 * dx and dW are the gradients of sum_t g_t loss_t; scale is 1 / (tokens that count in the whole batch) for the usual mean.
 *
 * A token whose label is negative does not count: its loss is 0, its row of dx is 0 and it adds nothing to dW, whatever its row
 * of x holds (NaN and infinities too) and whatever its dloss is.  A label of vocab or more is a mistake that only the device
 * can see: that loss is NaN, and the token adds no gradient.
 *
 * The scores z are never kept: the loss alone forms them in registers (HH_BF16) or for a block of tokens at a time; a step
 * holds them for a block of tokens in the workspace.
 *
 * HH_BF16: x, W, dx bfloat16; scores, statistics and losses fp32; dW fp32.  d enters the product for dx as bfloat16 (dx is rounded
 * to that at its end anyway) and the one for dW as a sum of two, which is within 2^-16 of each d: with scores of deviation 1.5 and
 * labels some 4 above them dW was 1.4e-6 to 2.2e-6 off the exact gradient of the given x and W (2-norm), where products in fp32 leave
 * 4e-7 to 8e-7 and one bfloat16 number would leave 2e-3.
 * HH_F32: everything fp32.
 * Both: a score's own rounding, an ulp of its size in fp32, moves its p by as much of itself; the label's d = g_t (p - 1) keeps the
 * rounding of p, up to 2^-22 g_t, also where p is nearly 1 and little else is left of d.
 *
 * Shapes: hidden a multiple of 64 (HH_BF16) or 8 (HH_F32), at most 32768; vocab 1 .. 262144, any; tokens >= 1, any; x below 2^31
 * bytes, W below 2^32 - 2^25 (HH_ERR_UNSUPPORTED_SHAPE otherwise).  The whole vocabulary is on this GPU; of a tensor-parallel share
 * of it see hh_head_share_fwd. */
typedef struct {
    int32_t hidden;   /* H */
    int32_t vocab;    /* V */
    int32_t tokens;   /* T */
    int32_t dtype;    /* hh_dtype */
} hh_head_cfg;

/* Bytes of workspace of hh_head_loss, hh_head_share_fwd and of hh_head_step, hh_head_share_bwd (either pointer may be NULL).
 * Host arithmetic only.  A step's workspace grows with the tokens until a block of them has 2 GiB of d or 2 GiB of copies of its rows of
 * x, whichever is first, beside 512 MiB of scores (HH_F32: d takes their place), 64 MiB of the products' partial sums and 17 MiB of
 * statistics: 4.6 GiB at most (HH_F32: 4.1 GiB), where hidden is about vocab.  A loss's is 65 MiB at most (HH_F32: 2.01 GiB, with the
 * scores of a block). */
int hh_head_sizes(const hh_head_cfg *cfg, size_t *loss_workspace_bytes, size_t *step_workspace_bytes);

/* loss[T] (fp32) of x [T, H] under the weight w [V, H] and labels[T]. */
int hh_head_loss(hh_ctx *ctx, const hh_head_cfg *cfg, const void *x, const void *w, const int64_t *labels,
                 float *loss, void *workspace, void *stream);

/* The loss and its gradients.  dloss: [T] fp32 or NULL.  dx [T, H] may be x; dw [V, H] fp32, added to where accumulate != 0. */
int hh_head_step(hh_ctx *ctx, const hh_head_cfg *cfg, const void *x, const void *w, const int64_t *labels,
                 const float *dloss, float scale, float *loss, void *dx, float *dw, int accumulate,
                 void *workspace, void *stream);

/* The same under tensor parallelism, or for a vocabulary in pieces: w holds words first .. first + vocab - 1, and labels count in the
 * whole vocabulary.  What the shares have to tell each other lies between the two calls and is not part of this library, as the
 * all-reduces of the layers are not:
 *     fwd:  lse[T] = log(sum over this share of exp z_tv),  picked[T] = z_t,label where the share has the label, otherwise 0
 *     outside, over the shares:  lse = log(sum exp lse_share),  loss = lse - sum picked
 *     bwd:  with that lse,  d_tv = g_t (exp(z_tv - lse_t) - [first + v = label(t)]);  dx is this share's partial sum, to be
 *           added over the shares,  dW (+)= d^T x
 * Every token with a label of 0 or more counts.  bwd forms the scores again (a third more products than hh_head_step).  lse is one fp32
 * number, rounded in each share and again outside: that moves a loss by up to 2^-23 |lse| and exp(z - lse) by as much of itself, where
 * hh_head_step keeps the largest score and the sum apart and loses nothing to large scores. */
int hh_head_share_fwd(hh_ctx *ctx, const hh_head_cfg *cfg, const void *x, const void *w, const int64_t *labels, int32_t first,
                      float *lse, float *picked, void *workspace, void *stream);
int hh_head_share_bwd(hh_ctx *ctx, const hh_head_cfg *cfg, const void *x, const void *w, const int64_t *labels, int32_t first,
                      const float *lse, const float *dloss, float scale, void *dx, float *dw, int accumulate,
                      void *workspace, void *stream);

/* Global gradient norm and clipping over n tensors of any sizes:
 *     norm = sqrt(sum of all g^2),  factor = min(1, max_norm / (norm + 1e-6)),  out = factor * g
 * out == NULL counts a tensor without a clipped copy; out may be g.  Squares are formed and added in fp64, so gradients of any
 * size can be summed.  A norm that is not finite gives the factor NaN.  Pointers need the alignment of their type
 * alone (16 bytes for all pointers of a tensor, or the same distance from it, is faster).  tensors is a HOST array, read during the call;
 * n may be 0, and so may a count, whose pointers are not looked at; a count is at most 2^34.
 * result: device, fp32: result[0] = norm, result[1] = factor. */
typedef struct {
    const void *g;    /* gradient, in `dtype` */
    void *out;        /* clipped copy in the same type, or NULL */
    int64_t count;    /* elements */
    int32_t dtype;    /* hh_dtype */
    int32_t reserved; /* 0 */
} hh_clip_tensor;
#define HH_CLIP_WORKSPACE_BYTES ((size_t)8192)
int hh_grad_clip(hh_ctx *ctx, int n, const hh_clip_tensor *tensors, float max_norm, float *result, void *workspace, void *stream);

/* One step of Adam with decoupled weight decay on n tensors:
 *     g' = factor * g,  m = beta1 m + (1 - beta1) g',  v = beta2 v + (1 - beta2) g'^2
 *     p = p - lr (m / (1 - beta1^step) / (sqrt(v / (1 - beta2^step)) + eps) + decay p)
 * in fp32, with constants formed in fp64.  factor: device, fp32, one value (result + 1 of hh_grad_clip: clipped gradients need
 * not be written and read again), or NULL for 1; a factor that is not finite leaves every tensor as it is, and that call
 * was no step: the next one has the same number.  A bfloat16 parameter has an fp32 master copy, which is p above, and receives p
 * rounded; an fp32 parameter is its own master copy (master NULL).  step counts from 1.
 * Pointers, tensors, n and counts as in hh_grad_clip. */
typedef struct {
    void *param;
    float *master;     /* fp32 master copy of a HH_BF16 parameter, NULL for a HH_F32 one */
    float *m, *v;
    const void *g;     /* gradient, in grad_dtype */
    int64_t count;     /* elements */
    float decay;       /* weight decay of this tensor (0 for norm gains, as a rule) */
    int32_t param_dtype, grad_dtype;
    int32_t reserved;  /* 0 */
} hh_adamw_tensor;
typedef struct {
    double lr, beta1, beta2, eps;
    int64_t step;      /* >= 1 */
} hh_adamw_cfg;
int hh_adamw_step(hh_ctx *ctx, const hh_adamw_cfg *cfg, int n, const hh_adamw_tensor *tensors, const float *factor, void *stream);

#ifdef __cplusplus
}
#endif
#endif /* HH_TRAIN_H */
