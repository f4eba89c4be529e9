/*
 * specsteer_loss.h -- C ABI of the losses over full-vocabulary logits on MI355X (gfx950): what trains
 * the specialist that drafts, on the logits in the layout that specsteer.h verifies them in.
 *
 *   specsteer_token_logprobs       log P(y) of given tokens, as a rollout or a frozen reference needs them
 *   specsteer_token_logprobs_grad  the gradient of any loss of those log-probs with respect to the logits
 *   specsteer_policy_loss          the clipped policy loss with a KL term, and its gradient
 *   specsteer_preference_loss      the loss of paired sequences' log ratios, and its gradient
 *
 * Logits are [B, T, V], vocabulary contiguous, row (b, t) scoring tokens[b][t]; P = Softmax(h / tau) over the
 * whole vocabulary, tau = params->temperature.  As in specsteer.h a sequence's rows lie before those of the next: stride_t >= V and
 * stride_b >= (T - 1) stride_t + V, with any gaps.  [T, B, V] logits, whose sequences interleave, are refused.  mask [B, T] says which positions count: the logits, tokens and
 * other inputs of a position that does not are never read, its outputs are 0 and so is its row of the gradient.
 *
 * Gradients are written, not accumulated: grad_logits has the logits' type, each element is rounded to it once.
 * grad_logits may be the logits themselves (same pointer, same strides), which then are replaced; any other
 * overlap of an output with an input is not allowed.
 *
 * Pointers, streams and errors are as in specsteer.h: all arrays are device memory but for the parameters,
 * nothing is allocated, owned or waited for, argument errors return before anything is enqueued and leave every
 * output untouched.  Where B * T is 0, arrays without elements may be NULL.  All calls may be captured into a graph.  Sums are formed in a fixed order: the same call
 * gives the same bits.
 *
 * Values.  A logit of -inf, or of the type's lowest value, masks a token: probability zero (the lowest value in a
 * whole row is a uniform row).  In a whole-vocabulary KL a token that the policy masks counts nothing, whatever
 * the reference says of it, and so does one whose P is far below what fp32 holds; another that only the reference
 * masks makes the row's KL and gradient not finite (with the lowest value, or about as large as that).
 * A token outside [0, V) at a position that counts, or a row whose logits are all -inf, has the log-prob NaN, and
 * so have the loss and the gradient rows that depend on it.  A given token of probability zero has the log-prob
 * -inf: the KL estimated from it is +inf, its pair's margin +inf or -inf, of which the loss is 0 or +inf, and NaN only
 * where both sequences of a pair hold one.  Weights that pass fp32 (of a huge grad_scale, say) make a row's
 * gradient not finite.  +inf and NaN among the logits are unspecified but never fault.
 * The same row's log-prob may differ in its last bits between calls of different kinds and numbers of rows.
 */
#ifndef SPECSTEER_LOSS_H
#define SPECSTEER_LOSS_H

#include "specsteer.h"

#ifdef __cplusplus
extern "C" {
#endif

#define SS_LOSS_MAX_LENGTH (1 << 20) /* largest T                */
#define SS_LOSS_MAX_ROWS (1 << 24)   /* largest B * T            */

typedef struct {
    int32_t batch;         /* B >= 0 (0 is a no-op but for losses, which are 0)                        */
    int32_t length;        /* T, 0..SS_LOSS_MAX_LENGTH                                                 */
    int32_t vocab;         /* V, 1..SS_MAX_VOCAB                                                       */
    int32_t dtype;         /* ss_dtype of the logits and of their gradient                             */
    int64_t stride_b;      /* element stride between sequences of the logits; 0 => length * stride_t;  */
                           /* at least (length - 1) * stride_t + vocab                                 */
    int64_t stride_t;      /* element stride between rows, at least vocab;    0 => vocab               */
    int64_t grad_stride_b; /* the same of grad_logits                                                  */
    int64_t grad_stride_t;
    float temperature;     /* tau; finite, > 0, and 1.45 / tau < 3e38                                     */
    float grad_scale;      /* what gradients are multiplied by (a loss scale, one over accumulated     */
                           /* steps); finite.  Losses are not scaled.                                  */
} ss_loss_params;

/* Bytes of device scratch (256-byte aligned) that each call needs for these params; 0 for invalid ones.  What lies
 * in it needs no initialisation and is garbage afterwards; calls that may overlap in time need distinct workspaces,
 * graphs that may be replayed at the same time among them. */
size_t specsteer_loss_workspace_bytes(const ss_loss_params *params);

/*
 * Log-probs of given tokens.
 *   logits    device, [B, T, V]
 *   tokens    device, [B, T] int32
 *   mask      device, [B, T] bytes, 0 for positions that do not count; or NULL: all do
 *   logprobs  device, [B, T] fp32 out: log P(tokens[b][t])
 *   stats     device, [B, T, 2] fp32 out, or NULL: what specsteer_token_logprobs_grad takes, a power of two E and the
 *             row's sum of exponentials over 2^E (for logits beyond 2^20, and temperatures beyond 10^+-12, their maximum m and
 *             minus the sum over exp(m / tau)); 0 and 1 at positions that do not count
 *   workspace, workspace_bytes, stream  as in specsteer.h
 */
ss_status specsteer_token_logprobs(const void *logits, const int32_t *tokens, const uint8_t *mask,
                                   const ss_loss_params *params, float *logprobs, float *stats,
                                   void *workspace, size_t workspace_bytes, void *stream);

/*
 * The gradient of a loss L of token log-probs:  dL/dh_v = g (1[v = y] - P(v)) / tau,  g = dL/d logprobs[b][t].
 *   stats          device, [B, T, 2] as specsteer_token_logprobs left it for these logits and temperature
 *   grad_logprobs  device, [B, T] fp32: g
 *   grad_logits    device, [B, T, V] out
 */
ss_status specsteer_token_logprobs_grad(const void *logits, const int32_t *tokens, const uint8_t *mask,
                                        const float *stats, const float *grad_logprobs,
                                        const ss_loss_params *params, void *grad_logits, void *stream);

/* The loss is the sum over the tokens that count, not their mean. */
#define SS_LOSS_SUM 1u
/* The loss is the mean over the sequences with tokens that count of their tokens' mean, not the mean over all tokens. */
#define SS_LOSS_SEQ_MEAN 2u
/* advantages is [B], one for all of a sequence's tokens, not [B, T]. */
#define SS_LOSS_SEQ_ADVANTAGES 4u

typedef struct {
    float clip_low;  /* the ratio is clipped to [1 - clip_low, 1 + clip_high]; finite, 0..1 */
    float clip_high; /* finite, >= 0                                                        */
    float kl_coef;   /* finite, >= 0; above 0 it takes a reference                          */
    uint32_t flags;  /* SS_LOSS_ bits, at most one of SUM and SEQ_MEAN                      */
} ss_policy_params;

/*
 * The clipped policy loss with a KL term.  With lp = log P(y), r = exp(lp - old), A the token's advantage:
 *     l = -min(r A, clip(r, 1 - clip_low, 1 + clip_high) A) + kl_coef * KL
 * averaged over the tokens that count (see the flags).  KL is
 *     exp(d) - d - 1, d = ref_logprobs - lp               if ref_logprobs is given (an estimate from the token drawn),
 *     sum_v P(v) (log P(v) - log Q(v)), Q = Softmax(ref_logits / tau)     if ref_logits is.
 * With kl_coef 0 the KL is written to kl only.
 *   ref_logits    device, [B, T, V] with the logits' type and strides, or NULL
 *   old_logprobs  device, [B, T] fp32, of the policy that drew the tokens
 *   ref_logprobs  device, [B, T] fp32, or NULL; not both references
 *   advantages    device, [B, T] or [B] fp32
 *   loss          device, 1 fp32 out; 0 if no token counts
 *   logprobs      device, [B, T] fp32 out, or NULL
 *   kl            device, [B, T] fp32 out, or NULL; needs a reference
 *   grad_logits   device, [B, T, V] out, or NULL: the loss alone
 */
ss_status specsteer_policy_loss(const void *logits, const void *ref_logits, const int32_t *tokens,
                                const uint8_t *mask, const float *old_logprobs, const float *ref_logprobs,
                                const float *advantages, const ss_loss_params *params,
                                const ss_policy_params *policy, float *loss, float *logprobs, float *kl,
                                void *grad_logits, void *workspace, size_t workspace_bytes, void *stream);

typedef struct {
    float beta;            /* finite                                                                   */
    float label_smoothing; /* 0..0.5: the share of pairs taken to be labelled the wrong way round      */
    uint32_t flags;        /* 0 or SS_LOSS_SUM: the sum over the pairs, not their mean                 */
} ss_preference_params;

/*
 * The preference loss of P = B / 2 pairs, sequence i preferred to sequence P + i (B even):
 *     margin_i = beta * ((sum_t lp - ref) of i  -  (sum_t lp - ref) of P + i)
 *     pair_loss_i = -(1 - label_smoothing) log s(margin_i) - label_smoothing log s(-margin_i),  s the logistic function
 * sums over the tokens that count, the loss the mean of the pairs'.
 *   ref_logprobs  device, [B, T] fp32, or NULL: 0
 *   loss          device, 1 fp32 out (0 for B = 0)
 *   pair_loss     device, [P] fp32 out, or NULL
 *   margin        device, [P] fp32 out, or NULL
 *   logprobs      device, [B, T] fp32 out, or NULL
 *   grad_logits   device, [B, T, V] out, or NULL: the loss alone
 */
ss_status specsteer_preference_loss(const void *logits, const int32_t *tokens, const uint8_t *mask,
                                    const float *ref_logprobs, const ss_loss_params *params,
                                    const ss_preference_params *preference, float *loss, float *pair_loss,
                                    float *margin, float *logprobs, void *grad_logits, void *workspace,
                                    size_t workspace_bytes, void *stream);

/* What a status of these calls means (the codes are those of specsteer.h). */
const char *specsteer_loss_status_string(int status);

#ifdef __cplusplus
}
#endif
#endif /* SPECSTEER_LOSS_H */
