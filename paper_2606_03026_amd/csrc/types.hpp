// Element types of the kernels that take more than one: widening to FP32,
// rounding (to nearest even) from it, and vectors of 8 elements.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "buffer.hpp"
#include "spike_types.h"

namespace spk {

typedef __bf16 bf16;
typedef _Float16 f16;
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef float f32x8 __attribute__((ext_vector_type(8)));
typedef float f32x8_a16 __attribute__((ext_vector_type(8), aligned(16)));  // in memory: 16-byte aligned
typedef int8_t i8x8 __attribute__((ext_vector_type(8)));

template <typename T> struct Vec8;
template <> struct Vec8<float> { typedef f32x8_a16 type; };
template <> struct Vec8<bf16> { typedef bf16x8 type; };
template <> struct Vec8<f16> { typedef f16x8 type; };
template <> struct Vec8<int8_t> { typedef i8x8 type; };

template <typename T>
__device__ inline f32x8 load8(const T* p)
{
    const typename Vec8<T>::type v = *reinterpret_cast<const typename Vec8<T>::type*>(p);
    return __builtin_convertvector(v, f32x8);
}

// v as a value of its own: without this the compiler may fold the FP32
// product before it and the rounding to F16 into one mixed-precision
// instruction, in some kernels and not in others.
template <typename T>
__device__ inline float in_fp32(float v)
{
    if constexpr (__is_same(T, f16))
        asm("" : "+v"(v));
    return v;
}

template <typename T>
__device__ inline void store8(T* p, f32x8 v)
{
    for (int e = 0; e < 8; ++e)
        v[e] = in_fp32<T>(v[e]);
    *reinterpret_cast<typename Vec8<T>::type*>(p) = __builtin_convertvector(v, typename Vec8<T>::type);
}

inline int type_bytes(int type)
{
    switch (type) {
    case SPIKE_TYPE_F32: case SPIKE_TYPE_I32: return 4;
    case SPIKE_TYPE_BF16: case SPIKE_TYPE_F16: return 2;
    case SPIKE_TYPE_I64: return 8;
    default: return 1;
    }
}

inline bool is_float_type(int type) { return type == SPIKE_TYPE_F32 || type == SPIKE_TYPE_BF16 || type == SPIKE_TYPE_F16; }

inline bool aligned_to(const void* p, uintptr_t a) { return ((uintptr_t)p & (a - 1)) == 0; }

}  // namespace spk
