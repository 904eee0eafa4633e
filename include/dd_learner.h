/*
 * dd_learner.h -- the learner's inner step on one NVIDIA B200 (sm_100a), part of libddmerge.
 *
 * Between two synchronisations a learner runs InnerOpt on the fragments that it received
 * (Algorithm 1): loss and gradient of its model, then an optimizer step that leaves the copy
 * theta_m which dd_merge_fragment reads.  This header declares the operators of that step
 * whose time matters on the device:
 *   - the gated feed-forward block, forward and backward, on the learner's bf16 weights;
 *   - the global norm of a list of gradient tensors, and clipping by it;
 *   - the AdamW step over a list of tensors, which applies the clip scale on the way and
 *     writes the bf16 copy that the merge reads.
 * The paper gives neither the model nor InnerOpt as formulas; the formulas below are fixed here.
 *
 * The conventions of dd_merge.h hold: borrowed buffers, [device] and [host] pointers, work
 * enqueued on the given stream without waiting, host arrays consumed before return, DD_OK or
 * a negative dd_error, conditions of the data reported through a device-side record and not
 * as errors, one context per host thread, and no two calls through one context overlapping
 * on the GPU.
 */
#ifndef DD_LEARNER_H
#define DD_LEARNER_H

#include "dd_merge.h"

#ifdef __cplusplus
extern "C" {
#endif

/* ---- gradient norm, clipping, AdamW over many tensors --------------------------------- */

/* dd_grad_record.status beside DD_STATUS_OK: the norm came out infinite or NaN (dd_grad_norm says from
 * which finite elements on). */
enum { DD_STATUS_NONFINITE = 4 };

/* Written by the device; readable by the host once the stream has been synchronised. */
typedef struct {
    float norm;         /* sqrt(norm_sq) */
    float scale;        /* min(1, max_norm / (norm + 1e-6)); 1 when status != DD_STATUS_OK */
    int32_t status;     /* DD_STATUS_OK or DD_STATUS_NONFINITE */
    uint32_t reserved;
    double norm_sq;     /* sum of the squares of every element */
} dd_grad_record;

/*
 * norm = sqrt(sum over all tensors and elements of g^2), and the clip scale for max_norm.
 * Squares and the sums over up to 34 elements are taken in float32, everything beyond in
 * float64, in a fixed order (repeated calls give the same bits).  Range: with every element below
 * 3e18 no sum overflows; one element past 1.8e19 makes the norm infinite (DD_STATUS_NONFINITE), as an
 * infinite element does.  norm_sq is within 34 x 2^-24 of itself plus 2^-149 for each element: squares
 * below float32's normal range (elements below 1.1e-19) lose bits, and those of elements below
 * 2.6e-23 count as 0.
 *
 *   grads     [host] count device pointers to contiguous tensors, aligned to their element
 *             (16-byte aligned tensors are read in 16-byte pieces)
 *   sizes     [host] count element counts, each at most 2^34; 0 is allowed (its pointer may
 *             be NULL)
 *   dtypes    [host] count dd_dtype values as bytes
 *   count     >= 0; lists of more than 256 tensors take one launch per 256
 *   max_norm  >= 0, may be infinite (scale 1)
 *   record    [device] 8-byte aligned, required
 *
 * The first norm, clip or recorded merge on a context allocates its workspace, which synchronises the
 * device: make one before a stream capture.  No later norm or clip, of however many tensors, allocates.
 * (A batched merge of many fragments may replace the workspace; graphs captured before then are not to
 * be replayed.)
 */
int dd_grad_norm(dd_ctx *ctx, const void *const *grads, const uint64_t *sizes, const uint8_t *dtypes,
                 int count, float max_norm, dd_grad_record *record, void *cuda_stream);

/*
 * dd_grad_norm, then out = scale * g, rounded to the tensor's type.  outs == NULL scales in
 * place; then nothing is read again or written when the scale is 1.  If the norm is not
 * finite (record status DD_STATUS_NONFINITE) nothing is written.
 *
 *   outs      [host] NULL or count device pointers, same sizes and types as grads; outs[i]
 *             may equal grads[i] but not overlap it otherwise, nor overlap another output
 *             (DD_ERR_ALIAS; the pairs (outs[i], grads[i]) are checked)
 */
int dd_clip_gradients(dd_ctx *ctx, void *const *grads, void *const *outs, const uint64_t *sizes,
                      const uint8_t *dtypes, int count, float max_norm, dd_grad_record *record,
                      void *cuda_stream);

/* AdamW's constants; step counts from 1. */
typedef struct {
    double lr, beta1, beta2, eps, weight_decay;
    uint64_t step;
} dd_adamw;

/*
 * One AdamW step with decoupled weight decay over a list of tensors, in one pass:
 *
 *   g  = scale * grad                                  (scale of `clip`; 1 without it)
 *   m  = beta1 m + (1 - beta1) g
 *   v  = beta2 v + (1 - beta2) g^2
 *   p  = p (1 - lr weight_decay) - lr (m / (1 - beta1^step)) / (sqrt(v / (1 - beta2^step)) + eps)
 *   copy = p rounded to bf16 (round to nearest even)
 *
 * Arithmetic and state are float32; the constants (1 - beta, 1 - beta^step, 1 - lr weight_decay)
 * are formed in float64 on the host and rounded once.  If clip->status is not DD_STATUS_OK nothing is
 * written: the step is skipped.
 *
 *   params, exp_avg, exp_avg_sq   [host] count device pointers to float32, updated in place
 *   grads     [host] count device pointers, types in dtypes, read only
 *   copies    [host] NULL, or count device pointers to bf16 (entries may be NULL)
 *   clip      [device] NULL, or the record that dd_grad_norm wrote earlier on the stream
 * Every pointer is aligned to its element; a tensor whose pointers all are 16-byte aligned
 * (copies and bf16 gradients 8-byte) moves in 16-byte pieces.  The buffers of one tensor
 * must not overlap one another (DD_ERR_ALIAS).
 */
int dd_adamw_step(dd_ctx *ctx, const dd_adamw *opt, float *const *params, const void *const *grads,
                  float *const *exp_avg, float *const *exp_avg_sq, void *const *copies,
                  const uint64_t *sizes, const uint8_t *dtypes, int count,
                  const dd_grad_record *clip, void *cuda_stream);

/* ---- gated feed-forward block ------------------------------------------------------------ */

/* a(g) = g sigmoid(g), or the tanh form of GELU, g sigmoid(2 sqrt(2/pi) (g + 0.044715 g^3)). */
typedef enum { DD_ACT_SILU = 0, DD_ACT_GELU_TANH = 1 } dd_activation;

/*
 * Sizes, row strides and weights of a block.  Matrices are bf16, row-major, rows contiguous;
 * strides are in elements and multiples of 8, base pointers 16-byte aligned (DD_ERR_ALIGNMENT),
 * 0 means the row length itself (which then has to be a multiple of 8).  tokens may be 0;
 * 1 <= d, f; every size and stride is below 2^30 (DD_ERR_TOO_LARGE).  What lies between a
 * row's end and the next row's start is neither read nor written.
 */
typedef struct {
    uint64_t tokens, d, f;
    uint64_t ld_x;          /* x, dx: tokens rows of d */
    uint64_t ld_y;          /* y, residual, dy: tokens rows of d */
    uint64_t ld_gate;       /* gate, up: tokens rows of f (not looked at when neither is given) */
    uint64_t ld_in;         /* w_gate, w_up and their gradients: f rows of d */
    uint64_t ld_down;       /* w_down and its gradient: d rows of f */
    const void *w_gate, *w_up, *w_down;     /* [device] bf16 */
    int32_t activation;                     /* dd_activation */
    uint32_t flags;                         /* 0; DD_DEBUG_EXPIRE_WAIT (test hook, as in dd_merge.h): the first
                                             * copies are made to wait for bytes that never come, so the call's
                                             * bounded waits expire, `status` says so and the context stays usable */
} dd_gated_ffn;

/*
 * Memory: the first call of either direction on a context allocates 256 KB per SM (38 MB on a B200)
 * for partial products, which it keeps; no later call allocates unless `hidden` / `scratch` is NULL
 * and has to grow.  Make the first call before a stream capture, and bring `hidden` / `scratch` to a
 * captured call: a graph that was captured with NULL is not to be replayed once the context's has grown.
 *
 * gate = x w_gate^T,  up = x w_up^T,  y = [residual +] (a(gate) * up) w_down^T
 *
 * Sums are float32; the product a(gate) * up is taken from the float32 gate and up and
 * rounded to bf16 once, because the second product reads it as a bf16 operand.
 *
 *   x         [device] bf16
 *   residual  [device] bf16 or NULL; may be y itself
 *   gate, up  [device] bf16 outputs, both or neither: what dd_gated_ffn_backward needs
 *   hidden    [device] scratch of tokens * (f rounded up to 8) bf16, 16-byte aligned, or NULL:
 *             the context allocates and keeps one (growing it synchronises the device; the
 *             largest call first, or a caller's buffer, keeps later calls free of that)
 *   y         [device] bf16
 *   status    [device] NULL or a word that the call sets to DD_STATUS_WAIT_LIMIT if a bounded
 *             wait inside a kernel gave up (outputs are then unspecified); never cleared
 * Outputs overlap neither one another nor an input, y == residual excepted (DD_ERR_ALIAS).  Matrices of
 * one stride may lie side by side in the rows of one buffer (gate and up as its halves).
 */
int dd_gated_ffn_forward(dd_ctx *ctx, const dd_gated_ffn *block, const void *x, const void *residual,
                         void *gate, void *up, void *hidden, void *y, int32_t *status, void *cuda_stream);

/*
 * Gradients of the block for the output gradient dy (the residual's gradient is dy itself):
 *
 *   dh = dy w_down;   dup = dh * a(gate);   dgate = dh * up * a'(gate)
 *   dx = dgate w_gate + dup w_up
 *   dw_gate = dgate^T x;   dw_up = dup^T x;   dw_down = dy^T (a(gate) * up)
 *
 * gate and up are the forward call's.  Sums are float32; dgate, dup and a(gate) * up are each
 * rounded to bf16 once, as operands of the products behind them.  dx is bf16.
 *
 *   dw_gate, dw_up, dw_down  [device] grad_dtype, strides ld_in and ld_down as the weights'
 *             (multiples of 8 elements in either type); with accumulate != 0 they are added to
 *   scratch   [device] 3 * tokens * (f rounded up to 8) bf16, 16-byte aligned, or NULL as above
 */
int dd_gated_ffn_backward(dd_ctx *ctx, const dd_gated_ffn *block, const void *x, const void *gate,
                          const void *up, const void *dy, void *dx, void *dw_gate, void *dw_up,
                          void *dw_down, dd_dtype grad_dtype, int accumulate, void *scratch,
                          int32_t *status, void *cuda_stream);

#ifdef __cplusplus
}
#endif
#endif /* DD_LEARNER_H */
