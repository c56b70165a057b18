/*
 * head_logits.h -- C ABI of what a serving loop does to logits before a token
 * is drawn from them: penalties for tokens that were there, biases, a mask.
 *
 * The output head gives n rows of V logits for each of S sequences: one for the
 * next token, or one for each drafted token and the one after them (head_draft.h, n =
 * G + 1).  For row j of sequence s and token v, with
 *
 *     count = how often v is among the sequence's tokens ids[n_prompt .. n_ids) and its
 *             first j drafts
 *     seen  = count > 0, or v is among ids[0 .. n_prompt)
 *
 * in this order, in FP32:
 *
 *     x = logits[s][j][v]
 *     x = x > 0 ? x / repetition[s] : x * repetition[s]      where seen
 *     x = x - frequency[s] * count                           where count > 0
 *     x = x - presence[s]                                    where count > 0
 *     x = x + bias[s][i]                                     where v = bias_ids[s][i]
 *     out[s][j][v] = x, or -infinity where mask[s][j] has no bit v
 *
 * rounded once to the logits' type.  A token named several times in bias_ids
 * has the last one's bias.  Tokens outside [0, V) count for nothing.  A mask
 * without any bit leaves a row of -infinity, which head_draft_verify answers with token -1.
 *
 * Data layout (DEVICE pointers; each input but logits may be NULL, and is then
 * left out):
 *   logits, out  [S][n] rows of V elements of `type` (SPIKE_TYPE_F32, BF16 or F16),
 *                ld_logits / ld_out elements apart.  out may be logits itself; otherwise
 *                it must not overlap an input.
 *   ids          int32 [S] rows of L tokens, ld_ids apart.
 *   n_ids        int32 [S]: how many of them there are, clamped to [0, L]; NULL: L.
 *   n_prompt     int32 [S]: how many of these are the prompt's, clamped to [0, n_ids]; NULL: none.
 *   drafts       int32 [S][n - 1].
 *   repetition, presence, frequency   float [S].
 *   bias_ids, bias   int32 and float [S][n_bias] (both or neither).
 *   mask         uint32 [S][n] rows of ceil(V / 32) words, ld_mask words apart: bit v % 32 of
 *                word v / 32 allows token v.
 * Pointers are aligned to their elements (16-byte accesses where pointers and
 * strides allow).  0 <= S <= LOGITS_MAX_S, 1 <= n <= LOGITS_MAX_N, 1 <= V <= LOGITS_MAX_V, 0 <= L <=
 * LOGITS_MAX_L, 0 <= n_bias <= LOGITS_MAX_BIAS.
 *
 * One kernel is enqueued on `stream`; no workspace, nothing is allocated, nothing waits, and
 * the call can be captured in a HIP graph.  Counts are whole numbers, so equal calls give
 * equal bits.  Errors as in spike_proj.h.
 */
#ifndef HEAD_LOGITS_H
#define HEAD_LOGITS_H

#include <stdint.h>

#include "spike_proj.h"
#include "spike_types.h"

#ifdef __cplusplus
extern "C" {
#endif

#define LOGITS_MAX_S 4096
#define LOGITS_MAX_N 32
#define LOGITS_MAX_V (1 << 30)
#define LOGITS_MAX_L (1 << 22)
#define LOGITS_MAX_BIAS (1 << 16)

int head_logits_adjust(const void *logits, int64_t ld_logits, int32_t type, int32_t S, int32_t n, int32_t V,
                       const int32_t *ids, int64_t ld_ids, int32_t L, const int32_t *n_ids, const int32_t *n_prompt,
                       const int32_t *drafts, const float *repetition, const float *presence, const float *frequency,
                       const int32_t *bias_ids, const float *bias, int32_t n_bias, const uint32_t *mask,
                       int64_t ld_mask, void *out, int64_t ld_out, void *stream);

#ifdef __cplusplus
}
#endif

#endif /* HEAD_LOGITS_H */
