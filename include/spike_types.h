/*
 * spike_types.h -- element types of the entry points that take more than one.
 *
 * Values of the narrower types are widened to FP32 before any arithmetic and
 * results are rounded once, to nearest even, when they are stored.
 */
#ifndef SPIKE_TYPES_H
#define SPIKE_TYPES_H

#define SPIKE_TYPE_F32 0
#define SPIKE_TYPE_BF16 1
#define SPIKE_TYPE_F16 2
#define SPIKE_TYPE_I8 3  /* codes with one FP32 scale per row (quantize.h) */

#define SPIKE_TYPE_I32 4 /* token ids */
#define SPIKE_TYPE_I64 5

#endif /* SPIKE_TYPES_H */
