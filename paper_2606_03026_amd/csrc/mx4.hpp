// Microscaled four-bit floating point (C ABI in include/quantize.h): the quantizer,
// and what the kernels that read codes share.
#pragma once

#include "types.hpp"

namespace spk {

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));

constexpr int kMxBlock = 32;  // elements that share an exponent

// The scale of an exponent byte as the conversions below read it: they take the exponent field of a float
// alone, 0 as 2^-127 and 255 as NaN.
__device__ inline float mx_scale(uint32_t byte) { return __uint_as_float(byte << 23); }

// Codes 2 J and 2 J + 1 of a register of eight, times their scale, rounded to two values of T.
template <typename T, int J>
__device__ inline uint32_t mx_pair(uint32_t codes, float scale)
{
    if constexpr (__is_same(T, f16))
        return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(codes, scale, J));
    else
        return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, J));
}

template <typename T>
__device__ inline u32x4 mx_eight(uint32_t codes, float scale)
{
    return u32x4{mx_pair<T, 0>(codes, scale), mx_pair<T, 1>(codes, scale), mx_pair<T, 2>(codes, scale), mx_pair<T, 3>(codes, scale)};
}

// --- quantizer -------------------------------------------------------------

// 8 elements on their way to codes.
template <typename T> struct MxEight {
    u32x4 v;  // 16-bit elements, as they were loaded

    __device__ inline void put(int e, T x) { v[e / 2] |= (uint32_t)__builtin_bit_cast(uint16_t, x) << (e % 2 * 16); }
    __device__ inline uint32_t largest() const  // the bits of the largest size, as FP32
    {
        uint32_t top = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t lo = v[i] & 0x7fffu, hi = v[i] >> 16 & 0x7fffu;
            top = top > lo ? top : lo;
            top = top > hi ? top : hi;
        }
        return __float_as_uint((float)__builtin_bit_cast(T, (uint16_t)top));
    }
    __device__ inline uint32_t codes(float scale) const
    {
        uint32_t c = 0;
        if constexpr (__is_same(T, f16)) {
            c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f16(c, __builtin_bit_cast(f16x2, (uint32_t)v[0]), scale, 0);
            c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f16(c, __builtin_bit_cast(f16x2, (uint32_t)v[1]), scale, 1);
            c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f16(c, __builtin_bit_cast(f16x2, (uint32_t)v[2]), scale, 2);
            c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f16(c, __builtin_bit_cast(f16x2, (uint32_t)v[3]), scale, 3);
        } else {
            c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(bf16x2, (uint32_t)v[0]), scale, 0);
            c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(bf16x2, (uint32_t)v[1]), scale, 1);
            c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(bf16x2, (uint32_t)v[2]), scale, 2);
            c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(bf16x2, (uint32_t)v[3]), scale, 3);
        }
        return c;
    }
};

template <> struct MxEight<float> {
    f32x4 v[2];

    __device__ inline void put(int e, float x) { v[e / 4][e % 4] = x; }
    __device__ inline uint32_t largest() const
    {
        uint32_t top = 0;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const uint32_t size = __float_as_uint(v[e / 4][e % 4]) & 0x7fffffffu;
            top = top > size ? top : size;
        }
        return top;
    }
    __device__ inline uint32_t codes(float scale) const
    {
        uint32_t c = 0;
        c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, v[0][0], v[0][1], scale, 0);
        c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, v[0][2], v[0][3], scale, 1);
        c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, v[1][0], v[1][1], scale, 2);
        c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, v[1][2], v[1][3], scale, 3);
        return c;
    }
};

// What eight codes stand for, as elements of T.
template <typename T>
__device__ inline MxEight<T> mx_values(uint32_t c, float scale)
{
    MxEight<T> r;
    if constexpr (__is_same(T, float)) {
        const f32x2 a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, scale, 0), b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, scale, 1);
        const f32x2 d = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, scale, 2), e = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, scale, 3);
        r.v[0] = f32x4{a[0], a[1], b[0], b[1]}, r.v[1] = f32x4{d[0], d[1], e[0], e[1]};
    } else {
        r.v = mx_eight<T>(c, scale);
    }
    return r;
}

struct QuantMx4Args {
    const void* x;
    int64_t ld_x;
    int M, K;
    uint32_t eights;  // groups of 8 elements of a row, whole blocks
    uint32_t units;   // M * eights
    uint8_t* codes;
    int64_t ld_codes;
    uint8_t* scales;
    int64_t ld_scales;
    void* values;
    int64_t ld_values;
};

// The larger of each lane's and its neighbour's under an XOR of the lane number's two lower bits.
template <int QUAD>
__device__ inline uint32_t quad_larger(uint32_t v)
{
    const uint32_t other = (uint32_t)__builtin_amdgcn_mov_dpp((int)v, QUAD, 0xf, 0xf, true);
    return v > other ? v : other;
}

constexpr int kQuantMx4Unroll = 4;

// A lane takes 8 elements, four lanes a block, whose largest goes round them; the
// conversions round to nearest even and saturate by themselves.  VEC: K is a multiple of 8 and rows of x and
// values start on 16-byte, rows of codes on 4-byte boundaries; else the 8 go in vectors at any address, but for a row's last.
// Bound by memory (57,344 x 1536 FP32 with values: 139 us for 751 MB, 5.4 TB/s; 57,000 x 1537 154 us, 353 element by element).
template <typename T, bool VEC>
__global__ __launch_bounds__(256) void k_quant_mx4(QuantMx4Args a)
{
    constexpr int U = kQuantMx4Unroll;
    MxEight<T> in[U];
    uint32_t row[U], v[U];
    const T* const x = static_cast<const T*>(a.x);
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const uint32_t i = blockIdx.x * (256u * U) + u * 256u + threadIdx.x;
        row[u] = i / a.eights, v[u] = i % a.eights;
        in[u] = MxEight<T>{};
        const int k = (int)v[u] * 8;
        if (i >= a.units || k >= a.K)
            continue;
        const T* const p = x + row[u] * a.ld_x + k;
        if constexpr (VEC) {
            in[u] = *reinterpret_cast<const MxEight<T>*>(p);
        } else if (k + 8 <= a.K) {
            __builtin_memcpy(&in[u], p, sizeof in[u]);
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e)
                if (k + e < a.K)
                    in[u].put(e, p[e]);
        }
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
        // (quad_perm 1,0,3,2 and 2,3,0,1)
        const uint32_t top = quad_larger<0x4e>(quad_larger<0xb1>(in[u].largest()));
        const bool live = blockIdx.x * (256u * U) + u * 256u + threadIdx.x < a.units;
        const bool finite = top < 0x7f800000u;
        const int exponent = (int)(top >> 23) - 2;
        const uint32_t byte = !finite ? 255u : exponent > 0 ? (uint32_t)exponent : 0u;
        const float scale = mx_scale(byte);
        const uint32_t c = finite ? in[u].codes(scale) : 0u;
        if (!live)
            continue;
        if (v[u] % 4 == 0)
            a.scales[row[u] * a.ld_scales + v[u] / 4] = (uint8_t)byte;
        const int k = (int)v[u] * 8;
        if (k >= a.K)
            continue;
        uint8_t* const to = a.codes + row[u] * a.ld_codes + v[u] * 4;
        T* const val = a.values ? static_cast<T*>(a.values) + row[u] * a.ld_values + k : nullptr;
        if constexpr (VEC) {
            *reinterpret_cast<uint32_t*>(to) = c;
            if (val)
                *reinterpret_cast<MxEight<T>*>(val) = mx_values<T>(c, scale);
        } else if (k + 8 <= a.K) {
            __builtin_memcpy(to, &c, 4);
            if (val) {
                const MxEight<T> r = mx_values<T>(c, scale);
                __builtin_memcpy(val, &r, sizeof r);
            }
        } else {
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (k + 2 * e < a.K)
                    to[e] = (uint8_t)(c >> (8 * e));
            if (val) {
                const MxEight<T> r = mx_values<T>(c, scale);
                const T* const each = reinterpret_cast<const T*>(&r);
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    if (k + e < a.K)
                        val[e] = each[e];
            }
        }
    }
}

}  // namespace spk
