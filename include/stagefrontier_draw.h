/*
 * stagefrontier_draw.h -- C ABI of libstagefrontier, third part: what a policy
 * step draws at random.
 *
 * The policy loss of stagefrontier_train.h takes tokens that were drawn, with
 * the log-probabilities that they had; these calls draw them: one token per row
 * of logits, or several at once from a smaller model's drafts, which are
 * accepted or replaced so that the target's distribution results.  The model
 * that is trained draws, too: which of its hidden values dropout keeps.
 *
 * Random numbers come by counter: a draw depends on the seed, the step, the call
 * site and its index, never on the launch, on how rows are shared among ranks,
 * or on what was drawn before.  So a backward pass makes a mask again instead of
 * storing it, a rank with a part of a tensor draws the part of its mask, and a
 * replayed graph draws anew when the step in device memory has been raised.
 * Tokens are decided in 64-bit arithmetic, by powers within 2^-39.7: they are
 * those of the definition, whatever the sizes, the strides and the split of the
 * work, but where a uniform number lies within about 2^-38 of a border between
 * two.  (A draft's acceptance: within 2^-38 of p_d relative to it.  A token from
 * what a target leaves of a draft's distribution: within 2^-37 / R, where R is the
 * share that is left, 2^-30 at least.)  Probabilities below 2^-700 of a row's
 * largest may count as 0.
 *
 * Conventions are those of stagefrontier.h: device pointers, asynchronous on
 * the caller's stream, buffers and workspaces allocated by the caller, no
 * mutable state in the library, SF_OK / SF_EINVAL / SF_EHIP, errors found on
 * the host returned before anything is enqueued.  A workspace may hold
 * anything before a call; its contents after one are unspecified, and two
 * calls that may run at the same time need one each.
 */
#ifndef STAGEFRONTIER_DRAW_H
#define STAGEFRONTIER_DRAW_H

#include "stagefrontier_train.h"

#ifdef __cplusplus
extern "C" {
#endif

/*
 * The generator is Philox4x32-10 (Salmon, Moraes, Dror and Shaw, "Parallel
 * random numbers: as easy as 1, 2, 3", SC 2011).  Its key is the seed; the four
 * words of its counter are
 *     low word of a block's number, its high word (bit 31: 1 for sf_uniform, 0
 *     for sf_dropout), the site, the low word of the step.
 * A key in device memory is int64[2]: the seed and the step, 8-byte aligned.
 * The site tells the calls of one step apart.  It is the caller's to choose;
 * calls of the same kind with the same seed, step, site and index draw the same.
 */

/*
 * sf_uniform -- uniform numbers in [0, 1), multiples of 2^-24:
 *     out[i] = 2^-24 floor(w / 2^8),  w = word (first + i) mod 4 of block
 *              (first + i) div 4.
 *
 *   key      device int64[2].
 *   site     any.
 *   first    index of out[0], >= 0; first + n <= 2^60.
 *   n        >= 0; 0 is a no-op.
 *   out      [n] float.
 *
 * Returns SF_OK, SF_EINVAL or SF_EHIP.
 */
int sf_uniform(const int64_t* key, uint32_t site, int64_t first, int64_t n, float* out,
               sf_stream_t stream);

/*
 * sf_dropout -- sets entries to 0 at random and scales the others, in one pass,
 * onto a residual or not:
 *     out[r][j] = residual[r][j] + (keep ? scale x[r][j] : 0)
 * The entry's index is e = first + r index_stride + j; it is kept where bits
 * 16 (e mod 2) and up of word (e mod 8) div 2 of block e div 8, 16 bits, are at
 * least t = floor(65536 p + 1/2), and scale = 65536 / (65536 - t), 0 where t =
 * 65536: p is taken to the nearest multiple of 2^-16, and the expectation is x,
 * but for the scale's rounding to a float.
 * The product is added in 32 bits with one rounding, and rounded once to the
 * output's type.  What is dropped counts as 0, also where x is not finite.
 *
 * The gradient is the same call: of x, sf_dropout of the output's gradient with
 * the same p, key, site, first and index_stride and no residual; of the
 * residual, the output's gradient itself.  A gradient is added to another by
 * giving that as the residual.
 *
 *   x               [N][x_stride] of type dtype, the first C entries of each
 *                   row used.
 *   out             [N][out_stride] of type out_dtype.  May be x or the
 *                   residual (same pointer, stride and type); else the memory
 *                   from its first to its last entry must hold none of theirs,
 *                   nor the gaps between their rows.  Entries from C on are
 *                   left alone.
 *   residual        [N][residual_stride] of type out_dtype, or NULL.
 *   dtype, out_dtype  SF_F32, SF_BF16 or SF_F16.
 *   N, C            N >= 0, C >= 0; with one of them 0 a no-op.  Each, and each
 *                   stride, at most 2^40.
 *   p               0 <= p <= 1.
 *   first           >= 0.
 *   index_stride    >= C: C where the rows are whole; the whole rows' length
 *                   where this is a part of their columns.  Every index stays
 *                   below 2^60.
 *
 * Returns SF_OK, SF_EINVAL or SF_EHIP.
 */
int sf_dropout(const void* x, int32_t dtype, int64_t N, int64_t C, int64_t x_stride, float p,
               const int64_t* key, uint32_t site, int64_t first, int64_t index_stride,
               const void* residual, int64_t residual_stride, void* out, int32_t out_dtype,
               int64_t out_stride, sf_stream_t stream);

/*
 * sf_token_sample -- draws a token of each row of logits by its distribution.
 * With z = inv_temperature * logits[i][:] and p = softmax(z),
 *     token = the lowest j with sum_{k <= j} p_k > uniform[i],
 *     logp  = log p_token.
 *
 *   logits, dtype, N, V, row_stride, inv_temperature: as for sf_token_logp.
 *   uniform          [N] float in [0, 1).  A row with a number outside takes no
 *                    part (an answer that has ended): it is not read, its token
 *                    is -1 and its logp 0.
 *   out_token        [N] int64.
 *   out_logp         [N] float, at most 0: rounded once, of a number within 2^-35
 *                    of log p, relative to it, and 2^-46 (2^-39 of rows of more
 *                    than 2^22 entries).
 *   workspace        sf_token_sample_workspace(dtype, N, V) bytes, 16-byte
 *                    aligned; may be NULL where that is 0.
 *
 * Logits of -inf are never drawn.  A row of nothing else has token -1 and
 * logp -inf; one that holds +inf or NaN has token -1 and logp NaN.  Of the
 * largest logits the first is drawn by a uniform number of 0 at a temperature
 * near 0.
 *
 * A uniform number is as fine as it is given.  By those of sf_uniform a token
 * comes in a multiple of 2^-24 of the draws, within 2^-24 of p_token (one less
 * probable than that in 2^-24 of them or never), while its logp is that of
 * p_token.  Returns SF_OK, SF_EINVAL or SF_EHIP.
 */
int sf_token_sample(const void* logits, int32_t dtype, int64_t N, int64_t V, int64_t row_stride,
                    const float* uniform, float inv_temperature, int64_t* out_token,
                    float* out_logp, void* workspace, int64_t workspace_bytes, sf_stream_t stream);

/* sf_token_sample_workspace -- bytes that sf_token_sample needs (0 where every
 * row is one workgroup's), -1 where an argument is out of range.  Host only. */
int64_t sf_token_sample_workspace(int32_t dtype, int64_t N, int64_t V);

/*
 * sf_draft_verify -- verifies drafted tokens against the target's probabilities
 * and draws one more of each sequence, over ragged sequences.  Sequence b has
 * n = seq_start[b+1] - seq_start[b] drafts, the rows s = seq_start[b] .. s + n - 1
 * of the draft's arrays, and n + 1 rows s + b .. s + b + n of the target's: the
 * last is the distribution after all drafts.  With p and q the softmax of a
 * target's and a draft's row, each by its own temperature, u the uniform number
 * of the target's row, and d the draft,
 *     a draft is accepted where u q_d < p_d, in turn until one is not;
 *     then a token is drawn with u' = the uniform number of the sequence's last
 *     target row, as by sf_token_sample, from
 *         max(p - q, 0) / sum max(p - q, 0)  of the row of the draft refused, or
 *         p of the last row with every draft accepted, and of a refused draft's
 *         row where that sum is below 2^-30 (p and q differ by rounding alone:
 *         such a draft was not drawn from q).
 * Without draft_logits every draft is taken as certain (looked up, or the
 * likeliest of a model): q_d = 1.
 * The tokens so emitted are distributed as if drawn from p one after the other,
 * where drafts were drawn from q, but for the steps of the uniform numbers (see
 * sf_token_sample).
 *
 *   target_logits    [D + B][target_stride], the first V entries of each row
 *                    used.  Aligned to the element size.
 *   draft_logits     [D][draft_stride] of the same type, or NULL.
 *   dtype            SF_F32, SF_BF16 or SF_F16.
 *   D, B, V          0 <= D < 2^31, 0 <= B < 2^31, 1 <= V <= 2^30.  B == 0 is a
 *                    no-op.
 *   target_stride, draft_stride  elements from one row to the next, >= V.
 *   draft            [D] int64.  One outside [0, V) is none: its sequence's
 *                    drafts end before it, and the token is drawn from p of its
 *                    row.  (So batches may be padded.)
 *   seq_start        [B+1] int64, ascending within [0, D].  (On the device, so
 *                    not checked; other values give unspecified results.)
 *   uniform          [D + B] float in [0, 1).
 *   inv_temperature, draft_inv_temperature  0 < . <= 2^100.
 *   out_accepted     [B] int64: drafts accepted.
 *   out_token        [D + B] int64: in a sequence's rows the accepted drafts,
 *                    the token drawn, then -1.
 *   out_logp         [D + B] float: log p of each, at the target's temperature, as
 *                    exact as sf_token_sample's; 0 where the token is -1.  Rows of no sequence are left as
 *                    they were.
 *   workspace        sf_draft_verify_workspace(dtype, D, B, V) bytes, 16-byte
 *                    aligned.
 *
 * Rows behind the draft that is refused may be read or not.
 *
 * A sequence ends without a token drawn (-1) at a row that is reached where the
 * uniform number, or that of the sequence's last row where a token is to be drawn,
 * lies outside [0, 1) (logp 0), the target's logits are all -inf (logp -inf), or
 * they or the draft's hold +inf or NaN (logp NaN).  A draft's
 * row of -inf alone has q = 0.  Returns SF_OK, SF_EINVAL or SF_EHIP.
 */
int sf_draft_verify(const void* target_logits, const void* draft_logits, int32_t dtype, int64_t D,
                    int64_t B, int64_t V, int64_t target_stride, int64_t draft_stride,
                    const int64_t* draft, const int64_t* seq_start, const float* uniform,
                    float inv_temperature, float draft_inv_temperature, int64_t* out_accepted,
                    int64_t* out_token, float* out_logp, void* workspace, int64_t workspace_bytes,
                    sf_stream_t stream);

/* sf_draft_verify_workspace -- bytes that sf_draft_verify needs, -1 where an
 * argument is out of range.  Host only. */
int64_t sf_draft_verify_workspace(int32_t dtype, int64_t D, int64_t B, int64_t V);

#ifdef __cplusplus
}
#endif

#endif /* STAGEFRONTIER_DRAW_H */
