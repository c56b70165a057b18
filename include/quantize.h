/*
 * quantize.h -- C ABI of the symmetric per-channel INT8 quantizer and
 * exporter, and of the quantizer to microscaled four-bit floating point.
 *
 * Operation (paper Sec. 2.3, "Quantization and Accumulation"): for a weight
 * matrix W [M][K] whose row m belongs to output channel m,
 *
 *     scale[m] = max(max_k |W[m][k]|, 1e-8) / 127
 *     Q[m][k]  = clip(round(W[m][k] / scale[m]), -127, 127)
 *
 * in binary32 arithmetic: the maximum is exact, 1e-8 is its nearest binary32
 * value, both divisions are correctly rounded, and round() takes ties to
 * even.  The floor keeps an all-zero row finite (its Q is all zero).
 * Results are bit-identical to that definition.  Non-finite weights give
 * unspecified (but finite, in range) codes.
 *
 * Layouts of Q (all pointers are DEVICE pointers):
 *   SPIKE_LAYOUT_ROW_MAJOR  Q[m*K + k]: the dense continuous-input kernels
 *                           (dense_proj.h).
 *   SPIKE_LAYOUT_COL_MAJOR  Q[k*M + m]: the spike-gated projections
 *                           (spike_proj.h's W, with N = M): the column of
 *                           input k is M contiguous bytes (Sec. 2.2).
 * W is float [M][K] row-major; scale is float [M], one per OUTPUT channel in
 * both layouts.  Scales are always computed along the output axis of the
 * logical [M][K] matrix, before any transposition, so the export defect the
 * paper withdraws (App. "Pure-INT4 Export Correction": scales taken after
 * transposing to [K][M]) cannot arise here.
 *
 * Sizes: 1 <= M, K <= 2^24 and M * K <= 2^31.  The call enqueues one or two
 * kernels on `stream` (a hipStream_t, NULL for the default stream) and returns; it
 * allocates nothing.  Q and scale must not overlap W.
 *
 * Errors: SPIKE_OK (0) or a negative code from spike_proj.h, with the
 * message in spike_proj_last_error(); arguments are validated before any HIP
 * call.
 */
#ifndef SPIKE_QUANTIZE_H
#define SPIKE_QUANTIZE_H

#include <stdint.h>

#include "spike_proj.h"
#include "spike_types.h"

#ifdef __cplusplus
extern "C" {
#endif

#define SPIKE_LAYOUT_ROW_MAJOR 0
#define SPIKE_LAYOUT_COL_MAJOR 1

int spike_quantize_int8(const float *W, int32_t M, int32_t K, int32_t layout, int8_t *Q, float *scale,
                        void *stream);

/* Host-only check of a stored scale tensor against its weight: for a logical
 * [M][K] weight quantized per output channel in groups of `group` inputs
 * (group = K: one scale per channel), the scales must have shape
 * [M][ceil(K / group)] (scale_cols = 1 for per-channel scales).  A tensor of
 * shape [K][ceil(M / group)] -- the same element count when M and K trade
 * places -- is reported as scales taken along the wrong axis (after a
 * transposition), the defect the paper withdraws.  Returns SPIKE_OK or
 * SPIKE_EINVAL with the reason in spike_proj_last_error(). */
int spike_check_scale_shape(int32_t M, int32_t K, int32_t group, int32_t scale_rows, int32_t scale_cols);

/* Microscaled four-bit floating point (the paper's INT4 format has groups of 32 inputs
 * with a scale each, App. "Pure-INT4 Export Correction"; here the scale is a power of two and a
 * value has an exponent of its own).  For each row of x [M][K] and each block of 32 of its
 * elements (the last may be shorter), with the block's largest size in [2^p, 2^(p + 1)):
 *
 *     scales[m][b] = e = max(p + 125, 0)              the block's scale is 2^(e - 127)
 *     codes[m][k]  = the level nearest to x[m][k] / 2^(e - 127)
 *
 * A level is a sign (bit 3 of its code) and one of 0, 0.5, 1, 1.5, 2, 3, 4, 6 (bits 0 to 2); a
 * tie goes to the even code, sizes above 6 go to 6, and the sign is x's, a zero's too.
 * The code of element k is in byte k / 2 of its row, the even one in the lower half; a last byte
 * of one code has zeros above it.  A block of zeros has e = 0.  A block with a NaN or an infinity
 * has e = 255, which stands for NaN throughout, and zeros for codes.
 * values (or NULL): [M] rows of K elements of x's type, what the codes stand for (exact: a
 * level times the scale of elements of that type is one).
 *
 * x: [M] rows of K elements of x_type (SPIKE_TYPE_F32, BF16 or F16), ld_x elements apart; codes:
 * rows of ceil(K / 2) bytes, ld_codes apart; scales: rows of ceil(K / 32) bytes, ld_scales apart; values:
 * ld_values elements apart.  Bytes between rows are left as they are.  Pointers are aligned to their elements; rows go as
 * 16-byte accesses where pointers, strides and K allow.  1 <= M, K <= 2^24, M * K <= 2^31;
 * M = 0 is nothing.  One kernel is enqueued on `stream`; values may be x itself, otherwise outputs must not
 * overlap each other or x. */
#define SPIKE_MX4_BLOCK 32

int spike_quantize_mx4(const void *x, int32_t x_type, int64_t ld_x, int32_t M, int32_t K, uint8_t *codes,
                       int64_t ld_codes, uint8_t *scales, int64_t ld_scales, void *values, int64_t ld_values,
                       void *stream);

#ifdef __cplusplus
}
#endif

#endif /* SPIKE_QUANTIZE_H */
