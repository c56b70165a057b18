/*
 * spike_clip.h -- C ABI of the common norm of a list of gradients and of its
 * clipping.
 *
 * A tuning step (spike_embed.h, dense_fused.h give its gradients) bounds the
 * length of the whole gradient before the weights move.  Over all elements g
 * of all n tensors:
 *
 *     norm   = sqrt(sum g^2)
 *     factor = min(1, max_norm / norm)        (1 where norm is 0, infinite or NaN)
 *     out    = factor * g
 *
 * Precision: squares and sums in 64 bits (no FP32 gradient overflows them),
 * in an order that depends on the sizes alone, so equal calls give equal bits;
 * the factor is rounded to FP32, products are FP32 and rounded once to the
 * tensor's type.  Where the norm is infinite or NaN, because a gradient is, out
 * is g unchanged, and the caller sees it in result.  A norm of finite gradients is finite in
 * 64 bits and clips by what it is there; beyond FP32's range result has infinity for it, beside its factor.
 *
 * spike_clip_create takes host arrays of n entries and keeps a table of them in
 * device memory; it reads no gradient, and the tensors stay the caller's and
 * have to outlive the handle.
 *   grads   DEVICE pointers to sizes[i] contiguous elements of types[i]
 *           (SPIKE_TYPE_F32, BF16 or F16), aligned to them; NULL where sizes[i] is 0.
 *   outs    DEVICE pointers, as grads, or NULL: all in place; an entry that is
 *           NULL or equal to its gradient is in place.  No out may overlap another out or another
 *           gradient; otherwise tensors may be given twice.
 *   result  DEVICE float [2]: norm and factor.
 * 0 <= n <= CLIP_MAX_TENSORS, 0 <= sizes[i], their sum up to 2^40.  max_norm: positive,
 * or +infinity (the norm alone; in place nothing is written then).
 *
 * Two kernels are enqueued on `stream` by spike_clip_forward; nothing is
 * allocated, nothing waits, and the call can be captured in a HIP graph
 * (max_norm is then part of it).  The workspace (spike_clip_workspace_bytes, 16-byte
 * aligned, no initial contents) is the caller's; calls that share one must not
 * overlap.  A handle belongs to the device that was current at its creation.
 * Errors as in spike_proj.h.
 */
#ifndef SPIKE_CLIP_H
#define SPIKE_CLIP_H

#include <stdint.h>

#include "spike_proj.h"
#include "spike_types.h"

#ifdef __cplusplus
extern "C" {
#endif

#define CLIP_MAX_TENSORS (1 << 20)

typedef struct spike_clip *spike_clip_t;

/* Synchronous.  On failure *out_handle is NULL. */
int spike_clip_create(const void *const *grads, void *const *outs, const int32_t *types, const int64_t *sizes, int32_t n,
                      spike_clip_t *out_handle);

/* Waits for the device and frees the handle (NULL: nothing). */
int spike_clip_destroy(spike_clip_t handle);

/* Workspace of spike_clip_forward; -1 for a null handle. */
int64_t spike_clip_workspace_bytes(spike_clip_t handle);

int spike_clip_forward(spike_clip_t handle, float max_norm, float *result, void *workspace, int64_t workspace_bytes,
                       void *stream);

#ifdef __cplusplus
}
#endif

#endif /* SPIKE_CLIP_H */
