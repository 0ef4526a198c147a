/*
 * stagefrontier_train.h -- C ABI of libstagefrontier, second part: the
 * numbers that a training step itself yields, beside its stage times.
 *
 * The frontier accounting of stagefrontier.h says where a step's time went
 * and runs inside the training loop without stopping it.  The step's own
 * numbers (the log-probabilities and the loss of a policy step, its KL term
 * and entropy, the gradient norm, entries that are not finite) are taken here
 * in the same manner: on the step's stream, without a host synchronisation
 * (which the accounting would show as exposed time of every rank) and in a
 * fixed order of summation.  Vectors are read from 128-byte boundaries, so that
 * order depends on where logits and gradients begin: equal inputs with equal
 * strides give equal bits on every rank where their addresses are equal modulo
 * 128, and may differ in the rounding of 32-bit sums (of 64-bit sums: in the
 * last rounding) elsewhere.  sf_policy_loss does not depend on the address, nor
 * sf_token_logp_grad but in rows that it sums itself.
 *
 * Conventions are those of stagefrontier.h: device pointers, asynchronous on
 * the caller's stream, buffers and workspaces allocated by the caller, no
 * mutable state in the library, SF_OK / SF_EINVAL / SF_EHIP, errors found on
 * the host returned before anything is enqueued.  A workspace may hold
 * anything before a call; its contents after one are unspecified, and two
 * calls that may run at the same time need one each.
 */
#ifndef STAGEFRONTIER_TRAIN_H
#define STAGEFRONTIER_TRAIN_H

#include "stagefrontier.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Element types of logits and gradients. */
enum {
    SF_F32 = 0,  /* IEEE 754 binary32 */
    SF_BF16 = 1, /* bfloat16          */
    SF_F16 = 2   /* IEEE 754 binary16 */
};

/*
 * sf_token_logp -- log-probability of the taken token, normaliser and
 * entropy of every row of logits, in one read of the logits.  With
 * z = inv_temperature * logits[i][:] and t = targets[i],
 *     lse  = log sum_j e^(z_j)
 *     logp = z_t - lse
 *     H    = - sum_j p_j log p_j,   p_j = e^(z_j - lse).
 * Arithmetic and sums are in 32 bits.  Exponents are taken relative to a
 * reference that no term of a sum passes by more than a few powers of two, and
 * that follows the row's maximum.
 *
 *   logits           [N][row_stride], the first V entries of each row used.
 *                    Aligned to the element size.
 *   dtype            SF_F32, SF_BF16 or SF_F16.
 *   N, V             0 <= N, 1 <= V <= 2^30.  N == 0 is a no-op.
 *   row_stride       elements from one row to the next, >= V.
 *   targets          [N] int64.  A row whose target lies outside [0, V) takes
 *                    no part: it is not read, and its outputs are 0.
 *   inv_temperature  0 < inv_temperature <= 2^100.
 *   out_logp         [N] float.
 *   out_lse          [N] float.
 *   out_entropy      [N] float, or NULL where the entropy is not wanted.
 *   workspace        sf_token_logp_workspace(dtype, N, V) bytes, 16-byte aligned;
 *                    may be NULL where that is 0.
 *
 * Logits of -inf have probability 0.  A row of nothing else has no
 * distribution: logp = lse = -inf, H = 0.  In any other row lse is held within
 * the largest floats, so that -inf says this alone.  A row that holds +inf or
 * NaN gives NaN.  Returns SF_OK, SF_EINVAL or SF_EHIP.
 */
int sf_token_logp(const void* logits, int32_t dtype, int64_t N, int64_t V, int64_t row_stride,
                  const int64_t* targets, float inv_temperature, float* out_logp, float* out_lse,
                  float* out_entropy, void* workspace, int64_t workspace_bytes,
                  sf_stream_t stream);

/* sf_token_logp_workspace -- bytes that sf_token_logp needs for N rows of V
 * logits of a type (0 where every row is one workgroup's), -1 where an argument
 * is out of range.  Host only. */
int64_t sf_token_logp_workspace(int32_t dtype, int64_t N, int64_t V);

/*
 * sf_token_logp_grad -- the gradient of sf_token_logp's outputs back to the
 * logits.  With g = grad_logp[i] and h = grad_entropy[i] (0 where NULL),
 *     out[j] = inv_temperature * (g ([j = t] - p_j) - h p_j (log p_j + H)).
 * log p_j = z_j - lse with lse as given while |lse| < 2^16, where its rounding is
 * a relative error of p of 2^-24 |lse|, up to 2^-9.  In a row with lse
 * beyond, whose logits lie far from 0, the kernel takes log p_j relative to the
 * row's maximum, with a sum of its own over the row; lse then only says so.
 *
 *   logits, dtype, N, V, row_stride, targets, inv_temperature: as for
 *                    sf_token_logp.
 *   lse              [N] float (out_lse of sf_token_logp).
 *   grad_logp        [N] float.
 *   entropy          [N] float (out_entropy), needed with grad_entropy only.
 *   grad_entropy     [N] float or NULL.
 *   out_grad         [N][out_row_stride] of the logits' type, rounded once to
 *                    nearest even; entries from V on are left alone.  May be
 *                    the logits themselves (same pointer and stride); must
 *                    not overlap them in any other way.
 *
 * Rows that take no part (target outside [0, V)), and rows with lse = -inf,
 * get zeros; they are not read.  Returns SF_OK, SF_EINVAL or SF_EHIP.
 */
int sf_token_logp_grad(const void* logits, int32_t dtype, int64_t N, int64_t V, int64_t row_stride,
                       const int64_t* targets, float inv_temperature, const float* lse,
                       const float* grad_logp, const float* entropy, const float* grad_entropy,
                       void* out_grad, int64_t out_row_stride, sf_stream_t stream);

/* How sf_policy_loss weighs a token. */
enum {
    SF_MEAN_TOKENS = 0,    /* 1 / (tokens that take part)                     */
    SF_MEAN_SEQUENCES = 1, /* 1 / (sequences with such a token) / (such tokens
                              of the token's sequence)                        */
    SF_SUM_TOKENS = 2      /* 1: the caller divides, e.g. by the count over
                              all ranks                                       */
};

/*
 * sf_policy_loss -- clipped policy loss with a KL term over ragged sequences,
 * and its gradient, in one call.  Per token, with A its advantage:
 *     d = logp - old_logp,  r = e^d
 *     surr = -min(r A, clip(r, 1 - clip_low, 1 + clip_high) A)
 *     x = ref_logp - logp,  kl = e^x - x - 1            (0 without ref_logp)
 *     loss = surr + kl_coef * kl
 * and over tokens, with w the reduction's weight times scale, rounded once,
 *     out_terms = { sum w loss, sum w surr, sum w kl, sum w [clipped] }
 *     out_grad  = d out_terms[0] / d logp.
 * A token is clipped (and passes no gradient through r) where A > 0 and
 * d > log(1 + clip_high), or A < 0 and d < log(1 - clip_low).  r and e^x are
 * held at the largest float, so an advantage of 0 stays 0.  Tokens are weighed
 * and summed in 64 bits, in a fixed order.
 *
 *   logp, old_logp   [N] float.
 *   ref_logp         [N] float or NULL.
 *   advantage        [N] float (advantage_per_token != 0) or [B] float.
 *   mask             [N] uint8 or NULL: tokens with 0 take no part, whatever
 *                    their other inputs hold; their gradient is 0.
 *   seq_start        [B+1] int64, ascending within [0, N]: sequence b holds
 *                    the tokens [seq_start[b], seq_start[b+1]).  Tokens
 *                    outside every sequence take no part.  (On the device,
 *                    so not checked; other values give unspecified results.)
 *   N, B             0 <= N <= 2^34 - 2^11, 0 <= B < 2^31; N == 0 or B == 0 gives
 *                    zeros.
 *   reduction        SF_MEAN_TOKENS, SF_MEAN_SEQUENCES or SF_SUM_TOKENS.
 *   scale            finite factor of every weight.
 *   clip_low         0 <= clip_low < 1.   clip_high  >= 0, finite.
 *   kl_coef          finite.
 *   out_terms        [4] float.
 *   out_grad         [N] float.
 *   workspace        sf_policy_loss_workspace(N, B) bytes, 16-byte aligned;
 *                    may be NULL where that is 0 (small inputs).
 *
 * With nothing taking part the terms and the gradient are 0.  Returns SF_OK,
 * SF_EINVAL or SF_EHIP.
 */
int sf_policy_loss(const float* logp, const float* old_logp, const float* ref_logp,
                   const float* advantage, int32_t advantage_per_token, const uint8_t* mask,
                   const int64_t* seq_start, int64_t N, int64_t B, int32_t reduction, float scale,
                   float clip_low, float clip_high, float kl_coef, float* out_terms,
                   float* out_grad, void* workspace, int64_t workspace_bytes, sf_stream_t stream);

/* sf_policy_loss_workspace -- bytes for N tokens in B sequences, -1 where one
 * is out of range.  Host only. */
int64_t sf_policy_loss_workspace(int64_t N, int64_t B);

/*
 * sf_grad_list_init -- lays out a list of gradient tensors for sf_grad_norm
 * and sf_grad_clip in host memory of the caller's, once for as long as the
 * tensors stay where they are.  It reads the arrays below before it returns
 * and touches no device memory; the list holds no resource to release.
 *
 *   list         host memory of sf_grad_list_bytes(n) bytes, 8-byte aligned.
 *   grads        host array of n device pointers, each aligned to its element
 *                size; dense tensors in any order of dimensions.  A pointer may
 *                be NULL where numel is 0.
 *   numel        host array of n element counts, >= 0, below 2^40 each and in
 *                all.
 *   dtype        host array of n types (SF_F32, SF_BF16, SF_F16; a list may
 *                mix them).
 *   n            0 <= n <= 2^20.
 *
 * Returns SF_OK or SF_EINVAL.  sf_grad_list_bytes returns -1 for an n out of
 * range.
 */
int64_t sf_grad_list_bytes(int32_t n);
int sf_grad_list_init(void* list, int64_t list_bytes, const void* const* grads,
                      const int64_t* numel, const int32_t* dtype, int32_t n);

/*
 * sf_grad_norm -- L2 norms of the gradients of a list, tensor by tensor and in
 * all, and how many entries of each are not finite; one read of the gradients.
 * Squares are taken and summed in 64 bits (no overflow for any finite input),
 * in a fixed order, and each norm is rounded once.
 *
 *   list           a list of sf_grad_list_init.
 *   out_norms      [n] float: norm of each tensor (0 for an empty one).
 *   out_total      [1] float: norm over all tensors (0 for an empty list).
 *   out_nonfinite  [n] int64: entries that are infinite or NaN.
 *   workspace      sf_grad_norm_workspace(list) bytes, 16-byte aligned.
 *
 * A tensor with an infinite entry has norm inf, one with a NaN NaN.  A job
 * that shards its gradients gathers out_total of every rank and hands all of
 * them to sf_grad_clip.  Returns SF_OK, SF_EINVAL or SF_EHIP.
 */
int sf_grad_norm(const void* list, float* out_norms, float* out_total, int64_t* out_nonfinite,
                 void* workspace, int64_t workspace_bytes, sf_stream_t stream);
int64_t sf_grad_norm_workspace(const void* list);

/*
 * sf_grad_clip -- scales the gradients of a list to a largest norm:
 *     norm = sqrt(sum_i norms[i]^2),  c = min(1, max_norm / (norm + eps))
 *     out = c * grad.
 * The norm and the quotient are in 64 bits, c is rounded to a float once.  The
 * product is a float, rounded, and for SF_BF16 and SF_F16 rounded again to the
 * type, each to nearest even.  The norm stays on the device: the host need not
 * wait for it.
 *
 *   list        the gradients.
 *   out_list    where the scaled gradients go: the same list (in place) or
 *               one of as many tensors of the same counts and types, none of
 *               which may overlap another or, but for being the same tensor,
 *               a gradient.
 *   norms       [m] device float, the norms of disjoint parts of the
 *               gradients: out_total of sf_grad_norm, or that of every rank.
 *   m           1 <= m <= 65536.
 *   max_norm    > 0, finite.     eps   >= 0, finite.
 *   status      device uint32 or NULL.  Where the norm is not finite the
 *               gradients are left (copied) as they are and SF_ERANGE is
 *               OR-ed into *status; the library never clears it.
 *
 * In place with c = 1 the gradients are neither read nor written.  A list of
 * n == 0 tensors is a no-op that launches nothing and leaves *status; a rank
 * without gradients that wants the status of the others lists one tensor of 0
 * entries.  Returns SF_OK, SF_EINVAL or SF_EHIP.
 */
int sf_grad_clip(const void* list, const void* out_list, const float* norms, int64_t m,
                 float max_norm, float eps, uint32_t* status, sf_stream_t stream);

#ifdef __cplusplus
}
#endif

#endif /* STAGEFRONTIER_TRAIN_H */
