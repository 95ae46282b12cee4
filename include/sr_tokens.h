/*
 * sr_tokens.h -- C ABI of the sr_gate library's operators on token ids (NVIDIA B200, sm_100a).
 *
 * sr_train.h begins at a policy's logits and ends at their gradient.  The calls here are what lies
 * between those and the token ids at both ends of the policy: the embedding of the tokens that go in,
 * with the table's gradient, and the adjustment of the logits that come out -- penalties for tokens
 * that were seen before, biases, and the mask of what a grammar or an environment allows -- with its
 * gradient.  Rollouts that were sampled from adjusted logits have to be scored and trained on
 * adjusted logits: `out` of sr_adjust_logits is what sr_token_logprob and sr_policy_loss_logits take,
 * and the gradient that these write is what sr_adjust_logits_backward takes.
 *
 * Conventions are those of sr_train.h (device pointers, the caller's buffers, checks before anything
 * is enqueued, SR_DTYPE_*, rows `pitch` elements apart).
 */
#ifndef SR_TOKENS_H_
#define SR_TOKENS_H_

#include <stddef.h>
#include <stdint.h>

#include "sr_gate.h"
#include "sr_train.h"

#ifdef __cplusplus
extern "C" {
#endif

/*
 * sr_adjust_logits -- y from x, for every row t and token v, in this order:
 *   seen[v]      v stands in the row's history;  c[v]: how often it stands there behind the prompt
 *   y = x;       where seen:   y = y / repetition[t] for y > 0, y * repetition[t] otherwise
 *                where c > 0:  y = y - frequency[t] c - presence[t]
 *                where v has a bias: y = y + bias;   where v is not allowed: y = -inf
 * in fp32, rounded once to the logits' type: an adjustment below half a step of a 16-bit type is lost (bf16 has steps of 0.125
 * between 16 and 32, where a penalty of 0.05 changes nothing); fp32 logits keep it.  What is neither seen, biased nor forbidden keeps its bits.
 * A token that is not allowed is -inf whatever stands there (a NaN for one), and a row may have nothing but such tokens.
 * Rows of logits and `out` on 16 bytes are fastest.  Rows of the two that begin at different distances from 16 bytes are handled
 * element by element and take several times as long, in the gradient too: with a padded pitch of the logits, give `out` the same.
 *
 *   logits         in  [n_rows][vocab] of type `dtype`, row t at element t * pitch
 *   history        in  [n_history] int32, the ids of all histories; NULL with n_history == 0
 *   history_start  in  [n_rows] int64 and history_len [n_rows] int32: row t's history is
 *                      history[history_start[t] .. + history_len[t]), prompt first.  Rows may share
 *                      one: a rollout that is scored as a whole gives all of its rows its start, and
 *                      lengths that grow by one (such rows one after the other are fastest).  Positions outside
 *                      0 .. n_history and ids below 0 do not count, ids >= vocab do not either and
 *                      set SR_STATUS_BAD_TARGET; a length below 0 is one of 0 and sets SR_STATUS_NEG_LEN; of a history
 *                      of 2^30 positions and more the first 2^30 - 1 count
 *   prompt_len     in  [n_rows] int32, how much of a history is prompt, or NULL: nothing (below 0 is 0)
 *   repetition, presence, frequency   in  [n_rows] fp32, each may be NULL: that penalty is left out.
 *                      repetition is > 0 and a normal number (16-bit logits are multiplied by its reciprocal).  All NULL: no histories are read and their arrays may be NULL
 *   bias_token     in  [n_bias] int32 and bias_value [n_bias] fp32: tokens with their biases.  Where a token stands in a
 *                      row's list more than once, the last one counts.  Ids below 0 or >= vocab as above
 *   bias_start     in  [n_rows] int64 and bias_len [n_rows] int32: row t's list is entries
 *                      bias_start[t] .. + bias_len[t], of 0 .. n_bias; rows may share one.  Of a list of more than 65535
 *                      entries the first 65535 count, and SR_STATUS_BAD_INDEX is set; a length below 0 as above.
 *                      bias_value NULL: no biases, the other three are not used
 *   allowed        in  [n_masks][mask_pitch] words of 32 bits: token v is allowed where bit v % 32 of word
 *                      v / 32 is set.  NULL: no masks.  mask_pitch >= ceil(vocab / 32)
 *   mask_row       in  [n_rows] int32, the mask of each row: below 0 none, and so >= n_masks, which sets
 *                      SR_STATUS_BAD_INDEX.  NULL: row t has mask t, and n_masks >= n_rows
 *   out            out [n_rows][vocab] of type `dtype`, row t at element t * out_pitch.  May be the logits
 *                      themselves (with out_pitch == pitch): then only vectors of 16 bytes in which something
 *                      changes are read and written.  Elements between vocab and the pitch are left as they are
 *   status         in/out 1 int32 of SR_STATUS_* bits; may be NULL
 */
int sr_adjust_logits(const void* logits, int32_t dtype, int32_t n_rows, int32_t vocab, int64_t pitch,
                     const int32_t* history, int64_t n_history, const int64_t* history_start,
                     const int32_t* history_len, const int32_t* prompt_len, const float* repetition,
                     const float* presence, const float* frequency, const int32_t* bias_token,
                     const float* bias_value, int64_t n_bias, const int64_t* bias_start,
                     const int32_t* bias_len, const uint32_t* allowed, int32_t n_masks, int64_t mask_pitch,
                     const int32_t* mask_row, void* out, int64_t out_pitch, int32_t* status, void* stream);

/*
 * sr_adjust_logits_backward -- the gradient of x from that of y:
 *   dx = 0 where v is not allowed;  where seen: dy / repetition[t] for x > 0, dy * repetition[t] otherwise;  dy elsewhere.
 * (The other penalties and biases are added: they do not change it.)
 *
 *   d_out          in  [n_rows][vocab] of type `dtype`, row t at element t * d_out_pitch
 *   logits         in  [n_rows][vocab] of the same type, as sr_adjust_logits had them, row t at element t * pitch;
 *                      read where a token was seen.  May be NULL where repetition is
 *   history ... mask_row   as above; repetition NULL: no histories are read
 *   d_logits       out [n_rows][vocab] of the same type, row t at element t * d_pitch.  May be d_out itself
 *                      (then only what changes is read and written) or the logits, with the same pitch
 */
int sr_adjust_logits_backward(const void* d_out, int32_t dtype, int32_t n_rows, int32_t vocab, int64_t d_out_pitch,
                              const void* logits, int64_t pitch, const int32_t* history, int64_t n_history,
                              const int64_t* history_start, const int32_t* history_len, const float* repetition,
                              const uint32_t* allowed, int32_t n_masks, int64_t mask_pitch,
                              const int32_t* mask_row, void* d_logits, int64_t d_pitch, int32_t* status,
                              void* stream);

/*
 * sr_embed_tokens -- out[t] = scale * table[tokens[t]], in fp32 and rounded to the type of `out`; zeros for a token below 0 (padding)
 * or >= vocab, which sets SR_STATUS_BAD_TARGET.
 *
 *   table      in  [vocab][width] of type `table_dtype`, row v at element v * table_pitch
 *   out        out [n_tokens][width] of type `dtype`, row t at element t * pitch.  The types are the same, or
 *                  the table's is SR_DTYPE_F32.  Rows on 16 bytes are fastest, and those on 8 or 4 next.
 *                  width is at most 2^24
 *   scale          finite in fp32
 */
int sr_embed_tokens(const void* table, int32_t table_dtype, int32_t vocab, int32_t width, int64_t table_pitch,
                    const int32_t* tokens, int32_t n_tokens, double scale, void* out, int32_t dtype,
                    int64_t pitch, int32_t* status, void* stream);

/*
 * sr_embed_tokens_backward -- the table's gradient: d_table[v] = scale * (sum over t with tokens[t] == v of
 * d_out[t]), for every row of it (+0 where no token took it), or, with accumulate, added to what stands there:
 * rows that no token took are then neither read nor written.
 *
 *   d_out      in  [n_tokens][width] of type `dtype`, row t at element t * pitch
 *   d_table    in/out [vocab][width] of type `table_dtype`, row v at element v * table_pitch; types as above
 *   workspace      device scratch of sr_embed_tokens_backward_workspace_bytes(n_tokens, vocab, width) bytes,
 *                  16-byte aligned; contents undefined before and after
 *
 * Tokens are sorted on the way; sums are in fp32, over t in ascending order within pieces of the sorted tokens whose
 * length depends on n_tokens and width alone, then over the pieces: the same call gives the same bits.  More than 4096 tokens are sorted by
 * a cluster of 16 CTAs, which a whole B200 holds; on a part of one that does not, the call returns SR_ERR_CUDA.
 */
int sr_embed_tokens_backward(const void* d_out, int32_t dtype, int32_t n_tokens, int32_t width, int64_t pitch,
                             const int32_t* tokens, int32_t vocab, double scale, void* d_table,
                             int32_t table_dtype, int64_t table_pitch, int32_t accumulate, int32_t* status,
                             void* workspace, size_t workspace_bytes, void* stream);
size_t sr_embed_tokens_backward_workspace_bytes(int32_t n_tokens, int32_t vocab, int32_t width);   /* host-only, pure */

#ifdef __cplusplus
}
#endif
#endif /* SR_TOKENS_H_ */
