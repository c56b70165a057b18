/*
 * dense_fused.h -- C ABI of the projection with INT8 or four-bit weights, with
 * bias, activation and residual in its epilogue, and of its gradient.
 *
 * Operation (paper Sec. 2.3, end of "Quantization and Accumulation": the
 * continuous-input projections, here with what a decoder block does to their
 * outputs; the runtime's activation is the exact GELU, Sec. 3):
 *
 *     z[b][m] = scale[m] * sum_k Q[m][k] x[b][k] + bias[m]
 *     y[b][m] = act(z[b][m]) + residual[b][m]
 *
 * and, with g[b][m] = dy[b][m] * act'(z[b][m]),
 *
 *     dx[b][k] = sum_m g[b][m] scale[m] Q[m][k],   dbias[m] = sum_b g[b][m]
 *
 * (the residual's gradient is dy; codes and scales are those of an export and
 * have none).  act is none, relu (derivative 0 at 0), gelu = z Phi(z) or
 * silu = z / (1 + exp(-z)).
 *
 * Precision.  A code is an integer of at most 8 bits, so BF16 and F16 hold it
 * exactly, and so are its products with BF16 or F16 activations in FP32.  FP32
 * activations of up to FUSED_FEW_ROWS rows are cut into BF16 parts that
 * add up to them exactly (three, and two more below 2^-110); those of more rows are scaled, row by row, by a power
 * of two and rounded to two F16 parts, which keep an element to 2^-23 of itself
 * or 2^-39 of its row's largest finite one, whichever is more (a caller that
 * needs every bit of rows with a wider range passes FUSED_FEW_ROWS at a time).
 * Each part is multiplied on the matrix cores.  All sums are FP32, in an order that depends
 * on the sizes alone; equal calls give equal bits (a row's bits may depend on
 * B).  z stays FP32 up to y; outputs are rounded once.  In the backward pass
 * g * scale is FP32 and enters the product in two such F16 parts, or of up to
 * FUSED_FEW_ROWS rows in these BF16 parts.  dbias is summed in FP32 from the
 * unrounded g.
 *
 * Four-bit weights (dense_fused_create_mx4; quantize.h states what codes and scales stand for) take the
 * place of scale[m] Q[m][k] in all of this; the same calls take the handle.  Its weights enter the product
 * as BF16 or F16 operands, each relative to a power of two that brings its output's largest block to
 * 2^13: exactly where that keeps them above 2^-127 (BF16 x, and FP32 x of up to FUSED_FEW_ROWS rows) or
 * 2^-24 (F16 x, and more rows of FP32 x: a weight is held to 2^-37 of its output's largest), and in the gradient to 2^-29
 * of its output's largest.  dense_fused_forward_mx4 takes rows of four-bit codes too, on matrix instructions
 * that scale the blocks; products are exact, sums FP32.  A block whose scale is 255 is NaN, and so is
 * every output whose sum has it.  Sums are of x times weights of size up to 2^16, so x above 2^100 may overflow them where z would not.
 *
 * Data layout (DEVICE pointers):
 *   codes, scales   of weights [M][K] or rows [B][K], as spike_quantize_mx4 writes them: rows of ceil(K / 2) and
 *             ceil(K / 32) bytes, ld_codes and ld_scales bytes apart, at any alignment; what lies behind
 *             element K is not read as part of it.
 *   Q         int8 [M][K] row-major, scale float [M] (as in dense_proj.h); read
 *             by create only, which lays them out for the matrix cores.
 *   x, dx     [B] rows of K elements, ld_x / ld_dx elements apart.
 *   y, dy, residual, pre   [B] rows of M elements, their ld_* apart, all of y_type.
 *   bias, dbias   float [M], or NULL.
 *   pre       forward: z is also written there; NULL: it is not.  Backward: z
 *             as the forward call wrote it; needed unless act is none.
 * Types F32, BF16 or F16, x_type for x and dx, y_type for the others.
 * Pointers are aligned to their elements; rows go as 16-byte accesses where
 * pointers, strides and sizes allow.  residual may be y itself; otherwise
 * outputs must not overlap inputs.
 *
 * Sizes: 1 <= K, M <= FUSED_MAX_DIM, their product, each rounded up to 64,
 * below 2^31; 0 <= B <= FUSED_MAX_B.
 *
 * A handle owns its copies of the weights (1 byte each, twice that with
 * DENSE_FUSED_BACKWARD; four-bit ones 9/16 of a byte and one more); calls on it only read them, so it may be used on
 * several streams at once.  forward and backward enqueue kernels on `stream`
 * (a hipStream_t, NULL for the default stream), allocate nothing, do not
 * synchronise and can be captured in a HIP graph.  The workspaces (their sizes
 * from the two queries below, 16-byte aligned, no initial contents) are the
 * caller's; calls that share one must not overlap.
 *
 * Errors: SPIKE_OK (0) or a negative code from spike_proj.h, with the message
 * in spike_proj_last_error(); arguments are validated before any launch.
 */
#ifndef DENSE_FUSED_H
#define DENSE_FUSED_H

#include <stdint.h>

#include "spike_proj.h"
#include "spike_types.h"

#ifdef __cplusplus
extern "C" {
#endif

#define DENSE_ACT_NONE 0
#define DENSE_ACT_RELU 1
#define DENSE_ACT_GELU 2
#define DENSE_ACT_SILU 3

#define DENSE_FUSED_BACKWARD 1 /* create: also lay the weights out for the gradient */

#define FUSED_MAX_DIM (1 << 20)
#define FUSED_MAX_B (1 << 22)
#define FUSED_FEW_ROWS 32 /* up to here forward needs no workspace */

typedef struct dense_fused *dense_fused_t;

/* Lay out Q [M][K] and scale [M] on the current device (synchronous: waits
 * for the device before and after).  On failure *out_handle is NULL. */
int dense_fused_create(const int8_t *Q, const float *scale, int32_t K, int32_t M, int32_t flags,
                       dense_fused_t *out_handle);

/* The same of four-bit weights [M][K]. */
int dense_fused_create_mx4(const uint8_t *codes, int64_t ld_codes, const uint8_t *scales, int64_t ld_scales, int32_t K,
                           int32_t M, int32_t flags, dense_fused_t *out_handle);

/* Waits for the device and frees the handle (NULL: nothing). */
int dense_fused_destroy(dense_fused_t handle);

int dense_fused_forward(dense_fused_t handle, const void *x, int32_t x_type, int64_t ld_x, int32_t B,
                        const float *bias, int32_t act, const void *residual, int64_t ld_residual, void *y,
                        int32_t y_type, int64_t ld_y, void *pre, int64_t ld_pre, void *workspace,
                        int64_t workspace_bytes, void *stream);

/* Workspace of dense_fused_forward for these rows; where it is 0 the workspace may be NULL:
 * always for up to FUSED_FEW_ROWS rows, and for 16-bit ones that start on 16-byte boundaries
 * with K a multiple of 8 unless their sums are split over workgroups, which depends on the
 * sizes.  -1 for a null handle or a size or type it refuses. */
int64_t dense_fused_forward_workspace_bytes(dense_fused_t handle, const void *x, int32_t x_type, int64_t ld_x,
                                            int32_t B);

/* dense_fused_forward of B rows of four-bit codes; the handle's weights are four-bit ones. */
int dense_fused_forward_mx4(dense_fused_t handle, const uint8_t *codes, int64_t ld_codes, const uint8_t *scales,
                            int64_t ld_scales, int32_t B, const float *bias, int32_t act, const void *residual,
                            int64_t ld_residual, void *y, int32_t y_type, int64_t ld_y, void *pre, int64_t ld_pre,
                            void *workspace, int64_t workspace_bytes, void *stream);

/* Its workspace for these rows, which may be NULL where it is 0: for up to FUSED_FEW_ROWS rows, and
 * for rows of a multiple of 128 elements whose codes start on 16-byte and scales on 4-byte boundaries unless
 * their sums are split over workgroups.  -1 for a null handle, one of INT8 weights or a size it refuses. */
int64_t dense_fused_forward_mx4_workspace_bytes(dense_fused_t handle, const uint8_t *codes, int64_t ld_codes,
                                                const uint8_t *scales, int64_t ld_scales, int32_t B);

/* Workspace of dense_fused_backward for B rows; -1 for a null handle or a size or type it refuses. */
int64_t dense_fused_workspace_bytes(dense_fused_t handle, int32_t B, int32_t y_type);

/* dx and dbias may each be NULL, not both. */
int dense_fused_backward(dense_fused_t handle, const void *dy, int32_t y_type, int64_t ld_dy, const void *pre,
                         int64_t ld_pre, int32_t act, int32_t B, void *dx, int32_t x_type, int64_t ld_dx,
                         float *dbias, void *workspace, int64_t workspace_bytes, void *stream);

#ifdef __cplusplus
}
#endif

#endif /* DENSE_FUSED_H */
