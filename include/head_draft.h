/*
 * head_draft.h -- C ABI of the verification of drafted tokens against the
 * target's probabilities.
 *
 * A cheap model drafts up to G tokens for each of S sequences; the target's
 * output head (dense_proj.h, head_verify.h) then gives logits for the G + 1
 * positions at once.  Per sequence, with T its temperature:
 *
 *     p_i = softmax(target_i / T), q_i = softmax(draft_i / T)       i = 0 .. G
 *     draft i is accepted iff uniform_i * q_i(d_i) < p_i(d_i) and every earlier one is
 *     j = number of accepted drafts
 *     r = max(p_j - q_j, 0); r = p_j after the last draft, and where p_j - q_j is positive nowhere
 *     next token = the v with the largest r(v) / noise(v), the lowest such v; -1 where none is positive
 *
 * With uniform_i uniform on [0, 1) and noise(v) exponential with mean one
 * (an exponential race: v wins with probability r(v) / sum r), the tokens are
 * distributed as the target's own samples.  The random numbers are inputs, so
 * the result is a function of the inputs alone.
 *
 *  - T = 0: p and q are one at the lowest index of the largest logit, zero
 *    elsewhere (a T that is not positive counts as 0); temperature NULL: T = 1.
 *  - draft NULL (the drafter gives tokens only): q_i is one at d_i.
 *  - A logit of -inf or NaN has probability zero; +inf logits share the whole
 *    probability equally.  A row without any other logit has probability zero
 *    throughout: its draft is refused, and its next token is -1.
 *  - A drafted token outside [0, V) has probability zero and is refused.
 *  - noise entries that are not positive, or so large that the quotient is zero,
 *    never win, nor do others in their place: r is as above.
 *
 * Precision: FP32, with the hardware's base-2 exponential and reciprocal (of
 * noise; within one unit in the last place); the sums of the exponentials are
 * taken per part of a row and joined in a fixed order, so equal calls give equal
 * bits.
 *
 * Data layout (DEVICE pointers):
 *   target       [S][G + 1] rows of V logits, ld_target elements apart.
 *   draft        [S][G] rows of V logits, ld_draft elements apart, or NULL.
 *   drafts       int32 [S][G].
 *   n_draft      int32 [S]: drafts of each sequence (clamped to [0, G]), NULL: G.
 *                Rows past a sequence's drafts are not read.
 *   uniform      float [S][G]; noise float [S] rows of V, ld_noise apart.
 *   temperature  float [S] or NULL.
 *   tokens       int32 [S][G + 1] out: the accepted drafts, the next token,
 *                then -1.
 *   n_accepted   int32 [S] out.
 *   accept       float [S][G] out or NULL: min(1, p_i(d_i) / q_i(d_i)) (q = 0:
 *                1 where p > 0), 0 past the sequence's drafts.
 *   prob         float [S][G + 1] out or NULL: p_i of each token in `tokens`,
 *                0 where that is -1.
 *   workspace    head_draft_workspace_bytes(S, G, V) bytes, 16-byte aligned,
 *                owned by the caller; no initial contents needed; calls that
 *                share one must not overlap.
 * logits_type: SPIKE_TYPE_F32, BF16 or F16, of target and draft.  0 <= S <=
 * DRAFT_MAX_S, 0 <= G <= DRAFT_MAX_G, 1 <= V <=
 * DRAFT_MAX_V; pointers aligned to their
 * elements (16-byte loads where pointers and strides allow).
 *
 * Two kernels are enqueued on `stream`; nothing is allocated, nothing waits,
 * and the call can be captured in a HIP graph.  Errors as in spike_proj.h.
 */
#ifndef HEAD_DRAFT_H
#define HEAD_DRAFT_H

#include <stdint.h>

#include "spike_proj.h"
#include "spike_types.h"

#ifdef __cplusplus
extern "C" {
#endif

#define DRAFT_MAX_S 4096
#define DRAFT_MAX_G 31
#define DRAFT_MAX_V (1 << 30)

/* Workspace of head_draft_verify; -1 for sizes the call refuses. */
int64_t head_draft_workspace_bytes(int32_t S, int32_t G, int32_t V);

int head_draft_verify(const void *target, int64_t ld_target, const void *draft, int64_t ld_draft, int32_t logits_type,
                      const int32_t *drafts, const int32_t *n_draft, const float *uniform, const float *noise,
                      int64_t ld_noise, const float *temperature, int32_t S, int32_t G, int32_t V, int32_t *tokens,
                      int32_t *n_accepted, float *accept, float *prob, void *workspace, int64_t workspace_bytes,
                      void *stream);

#ifdef __cplusplus
}
#endif

#endif /* HEAD_DRAFT_H */
