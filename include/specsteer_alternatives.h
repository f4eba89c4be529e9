/*
 * specsteer_alternatives.h -- C ABI of what rows of full-vocabulary logits say beside the log-probs of given tokens: the
 * entropy of each row and its likeliest tokens, on MI355X (gfx950).  Drafts' trees grow from them, a server answers with
 * them, a training step takes the entropy's gradient.
 *
 *   specsteer_token_alternatives       log-probs of given tokens, entropy and top alternatives, in one pass over the logits
 *   specsteer_token_alternatives_grad  the gradient of any loss of those log-probs and entropies
 *
 * Logits, masks, strides, temperatures, gradients, pointers, streams, workspaces and errors are as in specsteer_loss.h, whose
 * library holds these calls too.  Its values hold here as well, and for what is new:
 *   The entropy is -sum_v P(v) log P(v) in nats; a token of probability zero adds nothing.  Its error is absolute, about
 *   2^-22 for rows near certainty too.
 *   Alternatives come by decreasing logit, ties (-0 and 0 among them) by increasing token id.  A masked token (-inf, or the
 *   type's lowest value in a row that has others) is none: slots that no token is left for hold -1 and -inf, and so do all
 *   slots of a position that does not count.
 *   NaN among the logits is unspecified but never faults, as everywhere: such tokens are no alternatives.
 */
#ifndef SPECSTEER_ALTERNATIVES_H
#define SPECSTEER_ALTERNATIVES_H

#include "specsteer_loss.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Bytes of device scratch specsteer_token_alternatives needs; 0 for params or a topk out of range. */
size_t specsteer_token_alternatives_workspace_bytes(const ss_loss_params *params, int32_t topk);

/*
 *   tokens        device, [B, T] int32, or NULL: no log-probs
 *   topk          0..SS_MAX_TOPK; more than the vocabulary has are empty slots
 *   logprobs      device, [B, T] fp32 out, or NULL; needs tokens
 *   entropy       device, [B, T] fp32 out, or NULL
 *   top_tokens    device, [B, T, topk] int32 out; NULL only if topk is 0
 *   top_logprobs  device, [B, T, topk] fp32 out; NULL only if topk is 0
 *   stats         device, [B, T, 2] fp32 out, or NULL: as of specsteer_token_logprobs, whose gradient takes them too
 */
ss_status specsteer_token_alternatives(const void *logits, const int32_t *tokens, const uint8_t *mask,
                                       const ss_loss_params *params, int32_t topk, float *logprobs, float *entropy,
                                       int32_t *top_tokens, float *top_logprobs, float *stats, void *workspace,
                                       size_t workspace_bytes, void *stream);

/*
 * The gradient of a loss L of log-probs and entropies, g = dL/d logprobs[b][t] and k = dL/d entropy[b][t]:
 *     dL/dh_v = (g (1[v = y] - P(v)) - k P(v) (log P(v) + H)) / tau.
 *   stats, entropy  device, as specsteer_token_alternatives left them for these logits and temperature; entropy may be
 *                   NULL without grad_entropy
 *   grad_logprobs   device, [B, T] fp32: g, or NULL: 0; needs tokens
 *   grad_entropy    device, [B, T] fp32: k, or NULL: 0; not both NULL
 *   grad_logits     device, [B, T, V] out; may be the logits themselves
 */
ss_status specsteer_token_alternatives_grad(const void *logits, const int32_t *tokens, const uint8_t *mask,
                                            const float *stats, const float *entropy, const float *grad_logprobs,
                                            const float *grad_entropy, const ss_loss_params *params, void *grad_logits,
                                            void *stream);

#ifdef __cplusplus
}
#endif
#endif /* SPECSTEER_ALTERNATIVES_H */
