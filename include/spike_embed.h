/*
 * spike_embed.h -- C ABI of the embedding lookup and of its table's gradient.
 *
 * Lookup (the decoder's token embedding, paper Sec. 2.1; FP32 in Sec. 2.3's
 * runtime, or the INT8 codes and row scales the exporter writes for a tied
 * vocabulary head):
 *
 *     out[t][d] = scale * table[ids[t]][d]                (I8: scale * (row_scale[id] * code))
 *
 * Gradient of the table:
 *
 *     dtable[v][d] = scale * sum over t with ids[t] = v of grad[t][d]   (+ dtable[v][d] if accumulate)
 *
 * A token whose id lies outside [0, V) is padding: its row of `out` is zero
 * and it adds nothing to any gradient.
 *
 * Precision: FP32 arithmetic, one rounding when a value is stored.  The
 * gradient is a sum by sorted tokens: the tokens of a row are added in
 * ascending t, in runs that end at fixed places of the sorted list, and the
 * runs are joined in ascending order; the order depends on the ids alone, so
 * equal calls give equal bits.
 *
 * Data layout (DEVICE pointers):
 *   table      [V] rows of D elements, ld_table elements apart (ld_table >= D).
 *   row_scale  float [V] for SPIKE_TYPE_I8, else NULL.
 *   ids        int32 or int64 [T].
 *   out        [T] rows of D elements, ld_out elements apart.
 *   grad       [T] rows of D elements, ld_grad elements apart.
 *   dtable     [V] rows of D elements, ld_table apart.  Without `accumulate`
 *              every row is written (zeros where no token names it); with it
 *              only the rows that some token names are read and written.
 * Types: table F32, BF16, F16 or I8 (gradient: not I8); out, grad F32, BF16 or
 * F16.  Every pointer is aligned to its element; rows go as 16-byte accesses
 * where pointers, strides and D allow.  1 <= V <= EMBED_MAX_V, 1 <= D <=
 * EMBED_MAX_D, 0 <= T <= EMBED_MAX_T, T * D <= 2^35 for the gradient.  Outputs
 * must not overlap inputs.
 *
 * Nothing is allocated or retained and the calls do not synchronise: they
 * enqueue kernels on `stream` (a hipStream_t, NULL for the default stream) and
 * can be captured in a HIP graph.  The workspace of the gradient belongs to
 * the caller: spike_embed_workspace_bytes(T, D) bytes, 16-byte aligned, no
 * initial contents needed; calls that share one must not overlap.
 *
 * Errors: SPIKE_OK (0) or a negative code from spike_proj.h, with the message
 * in spike_proj_last_error(); arguments are validated before any HIP call.
 */
#ifndef SPIKE_EMBED_H
#define SPIKE_EMBED_H

#include <stdint.h>

#include "spike_proj.h"
#include "spike_types.h"

#ifdef __cplusplus
extern "C" {
#endif

#define EMBED_MAX_V (1 << 28)
#define EMBED_MAX_D 65536
#define EMBED_MAX_T (1 << 22)
#define EMBED_MAX_GRAD ((int64_t)1 << 35)

int spike_embed_forward(const void *table, int32_t table_type, const float *row_scale, int32_t V, int32_t D,
                        int64_t ld_table, const void *ids, int32_t id_type, int32_t T, float scale, void *out,
                        int32_t out_type, int64_t ld_out, void *stream);

/* Workspace of spike_embed_backward for T tokens and rows of D elements; -1
 * for sizes the call refuses. */
int64_t spike_embed_workspace_bytes(int32_t T, int32_t D);

int spike_embed_backward(const void *grad, int32_t grad_type, int64_t ld_grad, const void *ids, int32_t id_type,
                         int32_t T, int32_t V, int32_t D, float scale, int32_t accumulate, void *dtable,
                         int32_t table_type, int64_t ld_table, void *workspace, int64_t workspace_bytes, void *stream);

#ifdef __cplusplus
}
#endif

#endif /* SPIKE_EMBED_H */
