/*
 * dd_decoder.h -- the rest of a decoder's training step on one NVIDIA B200 (sm_100a), part of libddmerge.
 *
 * Beside the gated feed-forward block (dd_learner.h) a learner whose fragments are a decoder's layers
 * needs, between two synchronisations:
 *   - rotary positions on queries and keys, and the rotation back of their gradients;
 *   - attention over packed sequences, forward and backward;
 *   - the loss over the vocabulary and its gradients, without the logits ever being stored whole.
 * The paper gives no model; the formulas below are fixed here.
 *
 * The conventions of dd_merge.h and dd_learner.h hold: borrowed buffers, [device] and [host]
 * pointers, work enqueued on the given stream without waiting, DD_OK or a negative dd_error, conditions
 * of the data reported through a device-side word and not as errors, one context per host thread, and no
 * two calls through one context overlapping on the GPU.  Every sum is taken in a fixed order: repeated
 * calls give the same bits.
 */
#ifndef DD_DECODER_H
#define DD_DECODER_H

#include "dd_learner.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Beside DD_STATUS_WAIT_LIMIT in a call's status word: offsets that decrease, are negative or pass the
 * last token.  Nothing is written then. */
enum { DD_STATUS_BAD_OFFSETS = 5 };

/* One tensor of [tokens, heads, dim]: the elements of a head are contiguous, strides are in elements;
 * 0 stands for those of a contiguous tensor.  Tokens and heads may be in either order in memory, and
 * several tensors may share the rows of one buffer (a projection's queries, keys and values), one behind
 * the other or head by head. */
typedef struct {
    void *data;             /* [device] */
    uint64_t ld_token, ld_head;
} dd_heads;

/* ---- rotary positions -------------------------------------------------------------------- */

/*
 * For token t, pair i < rotary_dim / 2 and the angle w = positions[t] frequencies[i]:
 *
 *   a' = magnitude (a cos w - b sin w),  b' = magnitude (b cos w + a sin w)
 *
 * where (a, b) are the elements (i, i + rotary_dim / 2) of a head, or (2 i, 2 i + 1) with `interleaved`.
 * `inverse` turns by -w: with it the call takes the gradients of its results to those of its inputs.
 * Elements from rotary_dim on are copied.  Angles are formed in float64 and reduced to a part of a turn
 * there, the rest is float32, rounded once: beside that rounding a' and b' are within
 * magnitude (|a| + |b|) (2^-21 + 2^-51 |w|) of the formula's values.  Angles of up to 2^29 radians lose less
 * there than in float32; from 2^50 on little of an angle is left.
 *
 * Scaled contexts come in through `frequencies` and `magnitude`.
 *
 *   q, q_out  heads x dim; k, k_out kv_heads x dim, or k->data NULL and kv_heads 0.  An output may be its
 *             own input (same strides), but overlaps neither it nor any other tensor otherwise
 *   positions [device] int32, or int64 with positions_64; a token with a negative position is none:
 *             its rows are left as they are
 *   frequencies [device] rotary_dim / 2 float64, radians per position
 * tokens may be 0; tokens < 2^24, heads, kv_heads < 2^16, 1 <= dim <= 1024 (DD_ERR_TOO_LARGE), rotary_dim even,
 * 2 <= rotary_dim <= dim.  Data is aligned to its element; where pointers and strides allow it moves in
 * 16-byte pieces.
 */
typedef struct {
    uint64_t tokens, heads, kv_heads, dim, rotary_dim;
    dd_dtype dtype;
    int32_t interleaved, inverse, positions_64;
    float magnitude;
} dd_rotary;

int dd_rotary_apply(dd_ctx *ctx, const dd_rotary *rotary, const dd_heads *q, const dd_heads *k, const dd_heads *q_out,
                    const dd_heads *k_out, const void *positions, const double *frequencies, void *cuda_stream);

/* ---- attention ------------------------------------------------------------------------------ */

/*
 * Sequences lie end to end in the rows of one buffer: sequence s is the tokens offsets[s] .. offsets[s + 1]
 * - 1.  Query head h reads head h / (heads / kv_heads) of keys and values.  For tokens i, j of one
 * sequence (j <= i with `causal`):
 *
 *   s_ij = scale q_i . k_j,  lse_i = log sum_j exp(s_ij),  o_i = sum_j exp(s_ij - lse_i) v_j
 *
 * Tensors are bf16; sums, exponentials and lse are float32; the weights exp(s_ij - m), m within a factor of
 * 2^8 of the row's largest, are rounded to bf16 as operands of the second product (their sum is not).
 * Rows outside every sequence are neither read into a result nor written; what they hold, NaN included, does
 * not matter.  A NaN or infinity within a sequence may reach every token of that sequence.
 *
 *   dim       a multiple of 8 up to 128; strides multiples of 8, data 16-byte aligned (DD_ERR_ALIGNMENT)
 *   heads     a multiple of kv_heads; tokens < 2^31, heads < 2^16
 *   offsets   [device] sequences + 1 int32, non-decreasing, within 0 .. tokens; NULL: one sequence of all
 *             tokens (sequences is not looked at).  A sequence may be empty
 */
typedef struct {
    uint64_t tokens, heads, kv_heads, dim;
    uint64_t sequences;                     /* < 2^24 */
    const int32_t *offsets;
    float scale;                            /* finite, above 0 */
    int32_t causal;
    uint32_t flags;                         /* 0 or DD_DEBUG_EXPIRE_WAIT, as for dd_gated_ffn */
} dd_attention;

/* Bytes of `scratch` below, at most; 0 where none is needed, and for arguments that the calls refuse. */
uint64_t dd_attention_scratch_bytes(const dd_attention *attention, int backward);

/*
 *   q, o [tokens, heads, dim]; k, v [tokens, kv_heads, dim].  o overlaps no input
 *   lse       [device] heads x tokens float32 (natural logarithm), or NULL when no backward pass follows
 *   scratch   [device] 16-byte aligned, or NULL: the context allocates and keeps one (growing it
 *             synchronises the device; bring one to a captured call, as for dd_gated_ffn_forward)
 *   status    [device] NULL or a word that the call sets to DD_STATUS_BAD_OFFSETS or
 *             DD_STATUS_WAIT_LIMIT (outputs are then unspecified); never cleared
 */
int dd_attention_forward(dd_ctx *ctx, const dd_attention *attention, const dd_heads *q, const dd_heads *k, const dd_heads *v,
                         const dd_heads *o, float *lse, void *scratch, int32_t *status, void *cuda_stream);

/*
 * Gradients for the output gradient d_o, with o and lse as the forward call left them:
 *
 *   p_ij = exp(s_ij - lse_i),  dp_ij = d_o_i . v_j,  ds_ij = p_ij (dp_ij - d_o_i . o_i)
 *   dv_j = sum_i p_ij d_o_i,  dq_i = scale sum_j ds_ij k_j,  dk_j = scale sum_i ds_ij q_i
 *
 * with dk and dv summed over the query heads that share them.  p and ds are rounded to bf16 as operands.
 * A token that sees itself alone has ds = 0.  Outputs are bf16 and overlap nothing else.
 */
int dd_attention_backward(dd_ctx *ctx, const dd_attention *attention, const dd_heads *q, const dd_heads *k, const dd_heads *v,
                          const dd_heads *o, const float *lse, const dd_heads *d_o, const dd_heads *dq, const dd_heads *dk,
                          const dd_heads *dv, void *scratch, int32_t *status, void *cuda_stream);

/* ---- loss over the vocabulary ------------------------------------------------------------------ */

/*
 * Softmax cross entropy of logits z = hidden weight^T, which are formed tile by tile and never stored
 * whole:
 *
 *   lse_t = log sum_v exp(z_tv),  loss_t = lse_t - z_t,target
 *
 * A negative target is none: loss 0 and no gradient.  A target from `vocab` on is an error of the data:
 * loss NaN and no gradient.  The hidden row of a token without a target still takes part in products, with
 * weight 0, and has to be finite.  Matrices as in dd_learner.h: bf16, rows contiguous, strides in elements and
 * multiples of 8, 16-byte aligned, 0 meaning the row length.  tokens may be 0; 1 <= d, vocab; sizes and
 * strides < 2^30 (DD_ERR_TOO_LARGE).
 */
typedef struct {
    uint64_t tokens, d, vocab;
    uint64_t ld_hidden;                     /* hidden, dhidden: tokens rows of d */
    uint64_t ld_weight;                     /* weight, dweight: vocab rows of d */
    const void *weight;                     /* [device] bf16 */
    const int64_t *targets;                 /* [device] tokens */
    uint32_t flags;                         /* 0 or DD_DEBUG_EXPIRE_WAIT */
} dd_vocab_loss;

/* Bytes of `scratch` below; 0 for sizes that the calls refuse. */
uint64_t dd_vocab_loss_scratch_bytes(dd_ctx *ctx, const dd_vocab_loss *loss, int backward);

/*
 *   hidden    [device] bf16
 *   loss, lse [device] tokens float32 each
 *   scratch, status as above (the first call on a context allocates what dd_gated_ffn_forward's does)
 */
int dd_vocab_loss_forward(dd_ctx *ctx, const dd_vocab_loss *l, const void *hidden, float *loss, float *lse, void *scratch,
                          int32_t *status, void *cuda_stream);

/*
 * Gradients for dloss_t, the derivative by each token's loss:
 *
 *   g_tv = dloss_t (exp(z_tv - lse_t) - [v = target_t]);  dhidden = g weight;  dweight = g^T hidden
 *
 * g is rounded to bf16 as an operand of the products, for a piece of the vocabulary at a time; sums are
 * float32, those of dhidden over all pieces too.
 *
 *   dloss     [device] tokens float32
 *   dhidden   [device] bf16;  dweight [device] grad_dtype, with accumulate != 0 added to
 */
int dd_vocab_loss_backward(dd_ctx *ctx, const dd_vocab_loss *l, const void *hidden, const float *lse, const float *dloss,
                           void *dhidden, void *dweight, dd_dtype grad_dtype, int accumulate, void *scratch, int32_t *status,
                           void *cuda_stream);

#ifdef __cplusplus
}
#endif
#endif /* DD_DECODER_H */
