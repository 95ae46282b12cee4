/*
 * sr_train.h -- C ABI of the trainer's operators of the sr_gate library (NVIDIA B200, sm_100a).
 *
 * sr_gate.h decides which groups are cut and gives every rollout its advantage (Eq. 1).  The
 * calls here are what a training step does with them on the GPU: log-probabilities of the
 * tokens that were taken (the teacher-forcing pass of Appendix C.2) and their gradient, the
 * policy loss over the rollouts that were kept, the global gradient norm (Section 4.5 compares
 * it between runs) and clipping.
 *
 * Conventions are those of sr_gate.h: DEVICE pointers, every buffer the caller's, work enqueued
 * on `stream`, checks made before anything is enqueued.  Buffers of a call do not overlap
 * unless it says so.  All of them belong to the current device.  A workspace serves one call at a
 * time: calls that follow one another on a stream may share it, calls and captured graphs that may
 * overlap need one each.
 *
 * Logits are [n_tokens][vocab] of type `dtype` (SR_DTYPE_*), row t starting at element
 * t * pitch, pitch >= vocab; rows need no alignment beyond that of an element (16 bytes are
 * fastest).  Row t is the distribution that token t was drawn from: shifting a model's outputs
 * against its inputs is the caller's job.  targets[t] is that token; a negative target marks a
 * token that does not count (a prompt or an observation), and one >= vocab is treated the same
 * and sets SR_STATUS_BAD_TARGET.  Logits of tokens that do not count are not read.
 *
 * With z = x / temperature the distribution is p_j = exp(z_j) / sum exp(z).  A logit of -inf is
 * a token that cannot occur: p = 0, gradient 0, no part in the entropy.  A row with a NaN, a
 * +inf, or nothing but -inf gives NaN in its own outputs and no others.
 */
#ifndef SR_TRAIN_H_
#define SR_TRAIN_H_

#include <stddef.h>
#include <stdint.h>

#include "sr_gate.h"

#ifdef __cplusplus
extern "C" {
#endif

/* element types of logits and gradients */
#define SR_DTYPE_F32 0
#define SR_DTYPE_BF16 1
#define SR_DTYPE_F16 2

/* how sr_loss_weights shares the loss out */
#define SR_LOSS_SUM 0              /* every token counts `scale` */
#define SR_LOSS_TOKEN_MEAN 1       /* scale / tokens that count in the batch */
#define SR_LOSS_ROLLOUT_MEAN 2     /* mean over rollouts with tokens of the mean over their tokens, times scale */

/*
 * sr_token_logprob -- log p of the taken token of every row.
 *
 *   temperature        > 0 and finite (1e-30 .. 1e30)
 *   logp       out [n_tokens] fp32; +0 for tokens that do not count
 *   row_stats  out [n_tokens][2] fp32 or NULL: the largest logit M and S = sum exp((x - M) / temperature),
 *                  which the backward pass starts from (log p_j = (x_j - M) / temperature - log S);
 *                  zeros for tokens that do not count
 *   entropy    out [n_tokens] fp32 or NULL: -sum p log p (nats); +0 for tokens that do not count
 *   status     in/out 1 int32 of SR_STATUS_* bits; may be NULL
 */
int sr_token_logprob(const void* logits, int32_t dtype, int32_t n_tokens, int32_t vocab, int64_t pitch,
                     const int32_t* targets, double temperature, float* logp, float* row_stats,
                     float* entropy, int32_t* status, void* stream);

/*
 * sr_token_logprob_backward -- gradient of the logits from those of logp and entropy:
 *   d_logits_j = (d_logp ([j = target] - p_j) - d_entropy p_j (log p_j + entropy)) / temperature.
 *
 *   row_stats, entropy  as written by sr_token_logprob for the same logits; entropy is read
 *                       only where d_entropy is given and may be NULL otherwise
 *   d_logp     in  [n_tokens] fp32
 *   d_entropy  in  [n_tokens] fp32 or NULL
 *   d_logits   out [n_tokens][vocab] of the logits' type, row t at element t * d_pitch; zeros for
 *                  tokens that do not count.  May be the logits themselves (with d_pitch == pitch);
 *                  elements between vocab and the pitch are left as they are.
 */
int sr_token_logprob_backward(const void* logits, int32_t dtype, int32_t n_tokens, int32_t vocab,
                              int64_t pitch, const int32_t* targets, const float* row_stats,
                              const float* entropy, const float* d_logp, const float* d_entropy,
                              double temperature, void* d_logits, int64_t d_pitch, void* stream);

/*
 * sr_loss_weights -- the weight of a token of every rollout in the batch's loss.
 *
 * The batch holds n_groups * N rollouts back to back: rollout r (= g * N + i) owns tokens
 * row_start[r] .. row_start[r+1].  A token counts when its mask byte is non-zero (Appendix C.2:
 * only action tokens enter the loss) and its group is kept (Appendix C.1: a cut group is
 * skipped).  Weights are of the whole batch, so that chunks of it, and several epochs over it,
 * use the same ones.  A rollout without a token that counts gets +0.
 *
 *   row_start  in  [n_groups * N + 1] int64, non-decreasing
 *   mask       in  [n_tokens] uint8: positions outside 0 .. n_tokens do not count.  NULL: every token
 *                  between a rollout's row starts counts, wherever these lie, and n_tokens is not used
 *   drop_mask  in  [n_groups] uint8 or NULL: non-zero = cut (sr_gate's stop, for example)
 *   mode           SR_LOSS_*;  scale: finite in fp32
 *   weight     out [n_groups * N] fp32
 *   counts     out 2 int64 or NULL: tokens that count, rollouts with at least one
 *   workspace      device scratch of sr_loss_weights_workspace_bytes(n_groups * N) bytes, 16-byte
 *                  aligned; contents undefined before and after
 */
int sr_loss_weights(const int64_t* row_start, const uint8_t* mask, int32_t n_tokens,
                    const uint8_t* drop_mask, int32_t n_groups, int32_t N, int32_t mode, double scale,
                    float* weight, int64_t* counts, void* workspace, size_t workspace_bytes, void* stream);
size_t sr_loss_weights_workspace_bytes(int32_t n_rollouts);   /* host-only, pure */

/*
 * sr_policy_loss -- clipped policy loss with a KL term, and its gradient.
 *
 * For a token t of rollout r with rho = exp(logp - logp_old), A = adv[r], d = logp_ref - logp:
 *   gain_t = A min(rho, 1 + clip_high) for A > 0, A max(rho, 1 - clip_low) for A < 0, 0 for A = 0
 *   kl_t   = exp(d) - 1 - d
 *   loss   = sum_r weight[r] sum_{t in r that counts} (beta kl_t - gain_t)
 *   d loss / d logp_t = weight[r] (-A rho [not clipped] + beta (1 - exp(d)))
 * A factor of 0 leaves its term out whatever stands beside it, a NaN for one: A = 0 the gain, beta = 0
 * the KL term (of loss and gradient; the figures of rho and kl are sums without these factors).
 * A token counts when it lies in a rollout whose weight is not 0 and its mask byte is non-zero;
 * what stands in the arrays for the others is not used.
 *
 *   logp       in  [n_tokens] fp32, under the policy that is trained
 *   logp_old   in  [n_tokens] fp32 under the policy that the rollouts came from, or NULL: the same (rho = 1)
 *   logp_ref   in  [n_tokens] fp32 under the reference policy, or NULL: no KL term
 *   adv        in  [n_rollouts] fp32, weight in [n_rollouts] fp32 (sr_loss_weights)
 *   row_start  in  [n_rollouts + 1] int64, non-decreasing, relative to token 0 of the arrays given:
 *                  a chunk of a batch passes its row_start minus the chunk's first token, and
 *                  values below 0 or above n_tokens are fine
 *   mask       in  [n_tokens] uint8 or NULL
 *   clip_low, clip_high, beta   >= 0 and finite (beta in fp32)
 *   loss       out 1 fp32
 *   d_logp     out [n_tokens] fp32 or NULL; +0 for tokens that do not count.  May be logp itself.
 *   stats      out 4 fp32 or NULL: the weighted sums of gain, kl, [clipped] and rho
 *   workspace      device scratch of sr_policy_loss_workspace_bytes(n_tokens) bytes, 16-byte aligned
 *
 * Sums over tokens are in fp64, in an order that depends on the sizes alone: the same call
 * gives the same bits.
 */
int sr_policy_loss(const float* logp, const float* logp_old, const float* logp_ref, const float* adv,
                   const float* weight, const int64_t* row_start, int32_t n_rollouts,
                   const uint8_t* mask, int32_t n_tokens, double clip_low, double clip_high, double beta,
                   float* loss, float* d_logp, float* stats, void* workspace, size_t workspace_bytes,
                   void* stream);
size_t sr_policy_loss_workspace_bytes(int32_t n_tokens);      /* host-only, pure */

/*
 * sr_policy_loss_logits -- the same loss from logits, with the gradient of the logits: what
 * sr_token_logprob, sr_policy_loss and sr_token_logprob_backward give one after the other, without
 * their arrays in between.  A token counts when its target is one, its mask byte is non-zero and
 * it lies in a rollout whose weight is not 0.  It is
 * fastest where the rows of d_logits lie against 16 bytes as those of the logits do: in place, or
 * with pitches that differ by a multiple of 16 bytes.
 *
 *   logp       out [n_tokens] fp32; +0 for tokens that do not count
 *   d_logits   out as for sr_token_logprob_backward (may be the logits themselves)
 *   status     in/out 1 int32 of SR_STATUS_* bits; may be NULL.  SR_STATUS_TIMEOUT: CTAs that share a
 *              row have waited for one another for a second (microseconds are usual) and have given
 *              up; loss and stats are NaN then, status or not, and nothing else that the call wrote
 *              is to be used
 *   workspace      device scratch of sr_policy_loss_logits_workspace_bytes(n_tokens) bytes, 16-byte aligned
 */
int sr_policy_loss_logits(const void* logits, int32_t dtype, int32_t n_tokens, int32_t vocab, int64_t pitch,
                          const int32_t* targets, const float* logp_old, const float* logp_ref,
                          const float* adv, const float* weight, const int64_t* row_start,
                          int32_t n_rollouts, const uint8_t* mask, double clip_low, double clip_high,
                          double beta, double temperature, float* loss, float* logp, void* d_logits,
                          int64_t d_pitch, float* stats, int32_t* status, void* workspace,
                          size_t workspace_bytes, void* stream);
size_t sr_policy_loss_logits_workspace_bytes(int32_t n_tokens);   /* host-only, pure */

/*
 * sr_grad_norm -- the L2 norm of all gradients together (Section 4.5), squares summed in fp64 in
 * an order that depends on the sizes alone.  Gradients of a call are at most 2^31 - 1 pieces of 16 KB (each
 * begins a piece of its own): SR_ERR_BAD_SIZE above.
 *
 *   grads, counts, dtypes   HOST arrays of n_tensors: device pointer, number of elements (0 is
 *                           fine, the pointer may then be NULL) and SR_DTYPE_* of each tensor;
 *                           read during the call only
 *   norm       out 1 fp32
 *   workspace      device scratch of sr_grad_norm_workspace_bytes(n_tensors) bytes, 16-byte aligned
 */
int sr_grad_norm(const void* const* grads, const int64_t* counts, const int32_t* dtypes,
                 int32_t n_tensors, float* norm, void* workspace, size_t workspace_bytes, void* stream);
size_t sr_grad_norm_workspace_bytes(int32_t n_tensors);       /* host-only, pure */

/*
 * sr_clip_grads -- every gradient times min(1, max_norm / (norm + 1e-6)), with the norm as
 * sr_grad_norm left it (or as several GPUs have combined theirs).
 *
 *   norm       in  1 fp32.  When it is not finite nothing is scaled (out receives the gradients
 *                  as they are) and SR_STATUS_NONFINITE is set: the step is the caller's to skip.
 *   max_norm       >= 0 and finite in fp32
 *   out            HOST array of n_tensors device pointers, same types and sizes; an entry may be
 *                  the gradient's own pointer (in place), and NULL for the array means all are.
 *                  Apart from that no two buffers overlap: SR_ERR_OVERLAP.
 */
int sr_clip_grads(const void* const* grads, const int64_t* counts, const int32_t* dtypes,
                  int32_t n_tensors, const float* norm, double max_norm, void* const* out,
                  int32_t* status, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* SR_TRAIN_H_ */
