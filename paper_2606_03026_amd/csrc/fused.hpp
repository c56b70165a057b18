// INT8 projection with bias, activation and residual in its epilogue (C ABI in
// include/dense_fused.h), on the matrix cores.
//
// Weights are laid out once: for 16 outputs and 64 inputs, 1 KB in the order
// in which 64 lanes take it, lane 16 g + c holding output c's codes of inputs
// 8 g .. 8 g + 7 and 32 + 8 g .. 32 + 8 g + 7.  A 16-byte load then is the
// A operand of two v_mfma_f32_16x16x32 instructions once its codes are
// widened to the activations' type, whatever K and M are (zeros past them).
// The activations are the B operand, so a lane's four results are four
// neighbouring outputs of one row.
#pragma once

#include <type_traits>

#include "types.hpp"

namespace spk {

constexpr int kFusedTile = 16;  // outputs and rows of one matrix instruction
constexpr int kFusedStep = 64;  // inputs of one weight load

inline int64_t fused_pad(int64_t n, int64_t to) { return (n + to - 1) / to * to; }
inline int64_t fused_packed_bytes(int64_t n_out, int64_t n_in)
{
    return fused_pad(n_out, kFusedTile) * fused_pad(n_in, kFusedStep);
}

// Lays out Q [M][K] with its rows as outputs, or (TRANSPOSE) its columns; once per
// handle.  `eights`: rows start on 8-byte boundaries and K is a multiple of 8 (1536 ->
// 6144: 20 us byte by byte, 8 in eights).
template <bool TRANSPOSE>
__global__ __launch_bounds__(256) void k_fused_pack(const int8_t* __restrict__ Q, int K, int M, int8_t* __restrict__ P,
                                                    int64_t chunks, int eights)
{
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (i >= chunks)
        return;
    const int n_out = TRANSPOSE ? K : M, n_in = TRANSPOSE ? M : K;
    const int steps = (n_in + kFusedStep - 1) / kFusedStep;
    const int lane = i % 64;
    const int64_t piece = i / 64;
    const int64_t o = piece / steps * kFusedTile + lane % 16;
    const int64_t k0 = piece % steps * kFusedStep + lane / 16 * 8;
    union {
        int8_t b[16];
        u32x4 v;
    } w;
    if (!TRANSPOSE && eights) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int64_t k = k0 + 32 * h;
            const u32x2 v = o < n_out && k < n_in ? *reinterpret_cast<const u32x2*>(Q + o * K + k) : u32x2{};
            w.v[2 * h] = v[0], w.v[2 * h + 1] = v[1];
        }
        reinterpret_cast<u32x4*>(P)[i] = w.v;
        return;
    }
    for (int j = 0; j < 16; ++j) {
        const int64_t k = k0 + j % 8 + j / 8 * 32;
        w.b[j] = o < n_out && k < n_in ? (TRANSPOSE ? Q[k * K + o] : Q[o * K + k]) : 0;
    }
    reinterpret_cast<u32x4*>(P)[i] = w.v;
}

// --- values ----------------------------------------------------------------

// Operand types of the matrix instructions where rows are few: activations in BF16 parts, or F16 as they are.
template <typename XT> struct Operand { typedef bf16 type; };
template <> struct Operand<f16> { typedef f16 type; };

__device__ inline uint32_t high_halves(float lo, float hi)
{
    return __builtin_amdgcn_perm(__float_as_uint(hi), __float_as_uint(lo), 0x07060302u);
}

// Codes 2 i and 2 i + 1 of a register of four -> two operand values, exactly (a
// float that holds a code has its lower half zero).
template <typename OT>
__device__ inline uint32_t widen_pair(uint32_t w, int i)
{
    const float a = (float)(int8_t)(w >> (i * 16)), b = (float)(int8_t)(w >> (i * 16 + 8));
    if constexpr (__is_same(OT, f16)) {
        typedef __fp16 h2 __attribute__((ext_vector_type(2)));
        const h2 p = __builtin_amdgcn_cvt_pkrtz(a, b);
        return __builtin_bit_cast(uint32_t, p);
    } else {
        return high_halves(a, b);
    }
}

template <typename OT>
__device__ inline u32x4 widen_codes(uint32_t w0, uint32_t w1)
{
    return u32x4{widen_pair<OT>(w0, 0), widen_pair<OT>(w0, 1), widen_pair<OT>(w1, 0), widen_pair<OT>(w1, 1)};
}

// What of x is left after its upper 16 bits are taken off as a BF16 part; FIRST:
// x may be infinite, and nothing is left of it then (of what is left, never).
template <bool FIRST>
__device__ inline float below_bf16(float x)
{
    const float r = x - __uint_as_float(__float_as_uint(x) & 0xffff0000u);
    return FIRST && __builtin_isinf(x) ? 0.0f : r;
}

// Rows of FP32 values enter the product of many rows as two planes of F16 values: a row is
// scaled by the power of two that brings its largest size to [2^14, 2^15), then
// rounded, and what that leaves is rounded again for the second plane.
__device__ inline float largest(const float (&v)[8], float top)
{
#pragma unroll
    for (int e = 0; e < 8; ++e)
        top = fmaxf(top, __builtin_fabsf(v[e]));  // (leaves NaN out)
    return top;
}

// The power (2^126 at most: rows of subnormals are exact all the same; with an infinite
// element the one for the largest exponent, so that no other overflows) and its inverse.
struct RowPower {
    float factor, undo;
};

__device__ inline RowPower row_power(float top)
{
    const int shift = min(14 + 127 - min((int)(__float_as_uint(top) >> 23), 254), 126);
    return RowPower{__uint_as_float((uint32_t)(127 + shift) << 23), __uint_as_float((uint32_t)(127 - shift) << 23)};
}

// The largest over `waves` waves from wave `first` on, that this one is among.  s_top: one of
// two rows of LDS, taken in turn, so that the workgroup's one barrier is enough.
__device__ inline float largest_of_waves(float top, float (&s_top)[16], int first, int waves)
{
#pragma unroll
    for (int d = 32; d > 0; d /= 2)
        top = fmaxf(top, __shfl_xor(top, d));
    if (threadIdx.x % 64 == 0)
        s_top[threadIdx.x / 64] = top;
    __syncthreads();
    const int w = threadIdx.x % 16;
    top = s_top[first + (w < waves ? w : 0)];
#pragma unroll
    for (int d = 8; d > 0; d /= 2)
        top = fmaxf(top, __shfl_xor(top, d));
    return top;
}

// 8 values at p and p + plane.  Of an infinite one nothing is left for the second.
__device__ inline void put_planes(uint16_t* p, int64_t plane, const float (&v)[8], float factor)
{
    f16x8 hi, lo;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const float x = v[e] * factor;
        hi[e] = (f16)in_fp32<f16>(x);
        lo[e] = (f16)(__builtin_isinf(x) ? 0.0f : x - (float)hi[e]);
    }
    *reinterpret_cast<f16x8*>(p) = hi;
    *reinterpret_cast<f16x8*>(p + plane) = lo;
}

// 8 activations as they were loaded.
template <typename XT> struct Raw { u32x4 v; };
template <> struct Raw<float> { f32x4 v[2]; };

// Activations k .. k + 7 of rows of n; zeros past them.  VECX: n is a multiple
// of 8 and every row starts on a 16-byte boundary, so that a group of 8 lies
// inside a row or outside as a whole; the rows are read through a buffer
// resource that starts at `row0`, `at` elements from it.  Otherwise element by
// element.  No branches: loads stay in flight across the steps.
template <typename XT, bool VECX>
__device__ inline Raw<XT> load_raw(const XT* row0, __amdgpu_buffer_rsrc_t rsrc, int64_t at, int k, int n)
{
    Raw<XT> r;
    if constexpr (VECX) {
        const uint32_t off = k < n ? (uint32_t)(at + k) * (uint32_t)sizeof(XT) : kOutOfRange;
        if constexpr (sizeof(XT) == 4) {
            r.v[0] = __builtin_bit_cast(f32x4, __builtin_amdgcn_raw_buffer_load_b128(rsrc, off, 0, 0));
            r.v[1] = __builtin_bit_cast(f32x4, __builtin_amdgcn_raw_buffer_load_b128(rsrc, off, 16, 0));
        } else {
            r.v = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(rsrc, off, 0, 0));
        }
    } else {
        const XT* row = row0 + at;
        if constexpr (sizeof(XT) == 4) {
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float v = row[min(k + e, n - 1)];
                r.v[e / 4][e % 4] = k + e < n ? v : 0.0f;
            }
        } else {
            const uint16_t* p = reinterpret_cast<const uint16_t*>(row);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const uint32_t lo = p[min(k + 2 * e, n - 1)], hi = p[min(k + 2 * e + 1, n - 1)];
                r.v[e] = (k + 2 * e < n ? lo : 0u) | (k + 2 * e + 1 < n ? hi << 16 : 0u);
            }
        }
    }
    return r;
}

template <typename XT>
__device__ inline __amdgpu_buffer_rsrc_t rows_resource(const XT* row0)
{
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<XT*>(row0), 0, (int)kBufMaxBytes, kBufferFlags);
}

// Their NS operand parts.  Returns (in its lower half) what three parts leave of FP32 values:
// BF16's smallest step is 2^-133, FP32's 2^-149.
template <typename XT, int NS>
__device__ inline uint32_t split_raw(const Raw<XT>& r, u32x4 (&part)[NS])
{
    uint32_t left = 0;
    if constexpr (sizeof(XT) == 4) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            float a = r.v[i / 2][i % 2 * 2], b = r.v[i / 2][i % 2 * 2 + 1];
#pragma unroll
            for (int s = 0; s < NS; ++s) {
                part[s][i] = high_halves(a, b);
                if (s + 1 < NS) {
                    a = s == 0 ? below_bf16<true>(a) : below_bf16<false>(a);
                    b = s == 0 ? below_bf16<true>(b) : below_bf16<false>(b);
                }
            }
            left |= __float_as_uint(a) | __float_as_uint(b);
        }
    } else {
        part[0] = r.v;
    }
    return left & 0xffffu;
}

// That rest: the lower 16 bits of a subnormal value, as two operands of 8 bits in units of 2^-149.
__device__ inline void split_rest(const Raw<float>& r, u32x4 (&part)[2])
{
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        float v[2][2];
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            const float x = below_bf16<false>(below_bf16<true>(r.v[i / 2][i % 2 * 2 + e]));
            const uint32_t bits = __float_as_uint(x);
            v[0][e] = __builtin_copysignf((float)(bits & 0xff00u), x);
            v[1][e] = __builtin_copysignf((float)(bits & 0xffu), x);
        }
        part[0][i] = high_halves(v[0][0], v[0][1]);
        part[1][i] = high_halves(v[1][0], v[1][1]);
    }
}

template <typename OT>
__device__ inline f32x4 mfma16(u32x4 a, u32x4 b, f32x4 c)
{
    if constexpr (__is_same(OT, f16))
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
    else
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0,
                                                       0, 0);
}

// --- activations -----------------------------------------------------------

// Phi(-a) / exp(-a^2 / 2) for a >= 0 (half the scaled complementary error
// function of a / sqrt 2): a polynomial in t = 1 / (1 + 0.28 a), fitted to
// relative error 1.8e-7 over all a (least squares with weights raised where
// the error was largest, in double precision).  What it is multiplied with,
// exp2 of an argument rounded to FP32, adds about a^2 2^-24: the GELU of -3 to -6 is
// off by 2e-6 of itself, of -12 by 8e-6 (2e-9 and 2e-37), and below -13.2 it is 0.
__device__ inline float gauss_tail(float a)
{
    const float t = __builtin_amdgcn_rcpf(__builtin_fmaf(0.28f, a, 1.0f));
    float r = 0.024724291637539864f;
    r = __builtin_fmaf(r, t, -0.09361010789871216f);
    r = __builtin_fmaf(r, t, 0.09245535731315613f);
    r = __builtin_fmaf(r, t, -0.006472112610936165f);
    r = __builtin_fmaf(r, t, 0.0727858692407608f);
    r = __builtin_fmaf(r, t, 0.08362791687250137f);
    r = __builtin_fmaf(r, t, 0.10308506339788437f);
    r = __builtin_fmaf(r, t, 0.11169977486133575f);
    r = __builtin_fmaf(r, t, 0.11170385777950287f);
    return r * t;
}

// act(z) and act'(z) of W values.
template <int W>
__device__ inline void act_values(float (&z)[W], int act)
{
    switch (act) {
    case 1:
#pragma unroll
        for (int e = 0; e < W; ++e)
            z[e] = z[e] > 0.0f ? z[e] : z[e] == z[e] ? 0.0f : z[e];
        break;
    case 2:
#pragma unroll
        for (int e = 0; e < W; ++e) {
            const float tail = __builtin_amdgcn_exp2f(z[e] * z[e] * -0.72134752f) * gauss_tail(__builtin_fabsf(z[e]));
            z[e] *= z[e] < 0.0f ? tail : 1.0f - tail;
        }
        break;
    case 3:
#pragma unroll
        for (int e = 0; e < W; ++e)
            z[e] *= __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(z[e] * -1.44269504f));
        break;
    default: break;
    }
}

template <int W>
__device__ inline void act_slopes(float (&z)[W], int act)
{
    switch (act) {
    case 1:
#pragma unroll
        for (int e = 0; e < W; ++e)
            z[e] = z[e] > 0.0f ? 1.0f : z[e] == z[e] ? 0.0f : z[e];
        break;
    case 2:
#pragma unroll
        for (int e = 0; e < W; ++e) {
            const float x = __builtin_amdgcn_exp2f(z[e] * z[e] * -0.72134752f);
            const float tail = x * gauss_tail(__builtin_fabsf(z[e]));
            z[e] = __builtin_fmaf(z[e], x * 0.39894228f, z[e] < 0.0f ? tail : 1.0f - tail);
        }
        break;
    case 3:
#pragma unroll
        for (int e = 0; e < W; ++e) {
            const float sig = __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(z[e] * -1.44269504f));
            z[e] = sig * __builtin_fmaf(z[e], 1.0f - sig, 1.0f);
        }
        break;
    default:
#pragma unroll
        for (int e = 0; e < W; ++e)
            z[e] = 1.0f;
    }
}

// --- epilogue --------------------------------------------------------------

struct BiasArgs {
    const float* partial;
    int parts, M;
    float* dbias;  // NULL: none
};

struct FusedArgs {
    const int8_t* P;     // weights, laid out
    int n_out, n_in, steps;
    int w_steps;         // k_fused_tile: steps of an output's weights; walked again by the steps past them
    const void* x;
    int64_t ld_x;
    int64_t plane;       // elements between the planes of cut activations
    int B;
    const float* scale;  // NULL: one
    const float* row_scale;  // of rows that were scaled to F16 planes: what undoes that; NULL: one
    const float* bias;
    int act;
    const void* residual;
    int64_t ld_residual;
    void* y;
    int y_type;
    int64_t ld_y;
    void* pre;
    int64_t ld_pre;
    int vec_out;         // rows of y, residual and pre go in vectors of 8 (16 bytes at most)
    int out_tiles, row_tiles;
    int splits, split_steps;  // the steps go to `splits` workgroups, each writing its sums as FP32 rows at y
    int64_t split_stride;     // elements between their outputs
    BiasArgs bias_sums;       // workgroups behind the tiles' sum the parts of a bias gradient
};

// W elements at p: at once where `vec`, else the first n one by one.
template <typename T, int W>
__device__ inline void read_w(const T* p, float (&v)[W], bool vec, int n)
{
    typedef T tw __attribute__((ext_vector_type(W), aligned(W * sizeof(T) < 16 ? W * sizeof(T) : 16)));
    if (vec) {
        const tw r = *reinterpret_cast<const tw*>(p);
#pragma unroll
        for (int e = 0; e < W; ++e)
            v[e] = (float)r[e];
    } else {
#pragma unroll
        for (int e = 0; e < W; ++e)
            v[e] = e < n ? (float)p[e] : 0.0f;
    }
}

// (STREAM: past the caches)
template <typename T, int W, bool STREAM = false>
__device__ inline void write_w(T* p, const float (&v)[W], bool vec, int n)
{
    typedef T tw __attribute__((ext_vector_type(W), aligned(W * sizeof(T) < 16 ? W * sizeof(T) : 16)));
    if (vec) {
        tw r;
#pragma unroll
        for (int e = 0; e < W; ++e)
            r[e] = (T)in_fp32<T>(v[e]);
        if constexpr (STREAM)
            __builtin_nontemporal_store(r, reinterpret_cast<tw*>(p));
        else
            *reinterpret_cast<tw*>(p) = r;
    } else {
#pragma unroll
        for (int e = 0; e < W; ++e)
            if (e < n)
                p[e] = (T)in_fp32<T>(v[e]);
    }
}

template <typename T, int W, bool STREAM>
__device__ inline void put_outputs(const FusedArgs& a, int m, int64_t b, float (&z)[W], bool vec, int n, int64_t y_at)
{
    if (a.pre)
        write_w<T, W, STREAM>(static_cast<T*>(a.pre) + b * a.ld_pre + m, z, vec, n);
    act_values<W>(z, a.act);
    if (a.residual) {
        float r[W];
        read_w<T, W>(static_cast<const T*>(a.residual) + b * a.ld_residual + m, r, vec, n);
#pragma unroll
        for (int e = 0; e < W; ++e)
            z[e] += r[e];
    }
    write_w<T, W, STREAM>(static_cast<T*>(a.y) + y_at + b * a.ld_y + m, z, vec, n);
}

// Outputs m .. m + W - 1, a multiple of W: their scales and biases, read once
// for all rows that a lane stores.
template <int W>
struct OutputColumns {
    int m, n;      // n of them exist
    bool vec;
    float scale[W], bias[W];

    __device__ inline void load(const FusedArgs& a, int m_)
    {
        m = m_, n = min(W, a.n_out - m_), vec = a.vec_out && n == W;
        const int last = a.n_out - 1;
#pragma unroll
        for (int e = 0; e < W; ++e) {
            scale[e] = a.scale ? a.scale[min(m + e, last)] : 1.0f;
            bias[e] = a.bias ? a.bias[min(m + e, last)] : 0.0f;
        }
    }

    // y_at: elements from y's start to the rows
    template <bool STREAM = false>
    __device__ inline void store(const FusedArgs& a, int64_t b, float (&z)[W], int64_t y_at = 0) const
    {
        if (b >= a.B || n <= 0)
            return;
        if (a.scale) {
#pragma unroll
            for (int e = 0; e < W; ++e)
                z[e] *= scale[e];
        }
        if (a.bias) {
#pragma unroll
            for (int e = 0; e < W; ++e)
                z[e] += bias[e];
        }
        switch (a.y_type) {
        case SPIKE_TYPE_F32: return put_outputs<float, W, STREAM>(a, m, b, z, vec, n, y_at);
        case SPIKE_TYPE_BF16: return put_outputs<bf16, W, STREAM>(a, m, b, z, vec, n, y_at);
        default: return put_outputs<f16, W, STREAM>(a, m, b, z, vec, n, y_at);
        }
    }
};

// --- few rows --------------------------------------------------------------

// Up to 16 NB rows: a workgroup takes 16 MT outputs and all inputs, its WK
// waves sharing the 64-input steps; the waves' sums are joined in LDS.  Bound
// by the weights' bytes (1536 -> 57,344, one FP32 row: 18.8 us, 4.7 TB/s; BF16 16.8, 5.2),
// where these are few by latency (1536 -> 6144, one FP32 row: 5.0 us; 1536 -> 1536, 7 BF16
// rows: 3.0).  Asking whether three parts left anything costs 0 to 8% of an FP32 call (6144 ->
// 1536, 7 rows: 10.2 us without, 11.3).
// Rows that are not there cost no loads, only idle columns of the matrix instruction.
template <typename XT, int NS, int NB, int MT, int WK, bool VECX>
__global__ __launch_bounds__(64 * WK) void k_fused_rows(FusedArgs a)
{
    typedef typename Operand<XT>::type OT;
    constexpr int U = MT * NB >= 4 ? 1 : MT * NB >= 2 ? 2 : 4;  // steps in flight
    const int lane = threadIdx.x % 64, w = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
    const int g = lane / 16, c = lane % 16;
    const int tile0 = blockIdx.x * MT;
    const int64_t b0 = (int64_t)blockIdx.y * 16 * NB;
    const int tiles = (a.n_out + kFusedTile - 1) / kFusedTile;
    const XT* const x0 = static_cast<const XT*>(a.x) + b0 * a.ld_x;
    const __amdgpu_buffer_rsrc_t xr = rows_resource(x0), wr = weight_resource(a.P, kBufMaxBytes);
    static_assert(MT * NB <= WK, "a wave joins one tile's sums");
    // the waves that join sums ask for their columns first: these are back when the sums are
    OutputColumns<4> columns;
    if (w < MT * NB)
        columns.load(a, (tile0 + w / NB) * 16 + 4 * g);
    f32x4 acc[MT][NB];
#pragma unroll
    for (int t = 0; t < MT; ++t)
#pragma unroll
        for (int n = 0; n < NB; ++n)
            acc[t][n] = f32x4{};
    for (int s0 = w; s0 < a.steps; s0 += WK * U) {
        u32x4 wt[U][MT];
        Raw<XT> x[U][NB][2];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int s = s0 + u * WK;
#pragma unroll
            for (int t = 0; t < MT; ++t) {
                // (the vector offset is the one that the range check sees first)
                const bool live = s < a.steps && tile0 + t < tiles;
                const uint32_t piece = live ? ((uint32_t)(tile0 + t) * a.steps + s) * 1024u : 0u;
                wt[u][t] = __builtin_bit_cast(
                    u32x4, __builtin_amdgcn_raw_buffer_load_b128(wr, live ? lane * 16u : kOutOfRange, piece, 0));
            }
#pragma unroll
            for (int n = 0; n < NB; ++n) {
                const int b = 16 * n + c;
                const bool live = b0 + b < a.B && s < a.steps;
#pragma unroll
                for (int h = 0; h < 2; ++h)
                    x[u][n][h] = load_raw<XT, VECX>(x0, xr, min((int64_t)b, a.B - 1 - b0) * a.ld_x,
                                                    live ? s * kFusedStep + 32 * h + 8 * g : a.n_in, a.n_in);
            }
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (s0 + u * WK >= a.steps)
                break;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                u32x4 wo[MT];
#pragma unroll
                for (int t = 0; t < MT; ++t)
                    wo[t] = widen_codes<OT>(wt[u][t][2 * h], wt[u][t][2 * h + 1]);
#pragma unroll
                for (int n = 0; n < NB; ++n) {
                    u32x4 part[NS];
                    const uint32_t left = split_raw<XT, NS>(x[u][n][h], part);
#pragma unroll
                    for (int p = 0; p < NS; ++p)
#pragma unroll
                        for (int t = 0; t < MT; ++t)
                            acc[t][n] = mfma16<OT>(wo[t], part[p], acc[t][n]);
                    if constexpr (NS == 3) {
                        if (__builtin_expect(__any(left != 0), 0)) {  // (values below 2^-110 only)
                            u32x4 rest[2];
                            split_rest(x[u][n][h], rest);
#pragma unroll
                            for (int t = 0; t < MT; ++t)
                                acc[t][n] += mfma16<OT>(wo[t], rest[0], mfma16<OT>(wo[t], rest[1], f32x4{})) * 0x1p-149f;
                        }
                    }
                }
            }
        }
    }
    __shared__ f32x4 s_sum[WK][MT * NB][64];
#pragma unroll
    for (int t = 0; t < MT; ++t)
#pragma unroll
        for (int n = 0; n < NB; ++n)
            s_sum[w][t * NB + n][lane] = acc[t][n];
    __syncthreads();
    if (w >= MT * NB)
        return;
    f32x4 sum = s_sum[0][w][lane];
#pragma unroll
    for (int v = 1; v < WK; ++v)
        sum += s_sum[v][w][lane];
    const int64_t b = b0 + w % NB * 16 + c;
    float z[4] = {sum[0], sum[1], sum[2], sum[3]};
    columns.store(a, b, z);
}

// dbias from its parts (the first 256 threads of a workgroup: 64 outputs, a quarter of
// the parts per wave; s_sum: 256 floats of LDS).  Beside a product it is hidden; alone
// 16 parts of 6144 take 2.8 us, 157 of 12,000 (7.5 MB) 5.2.
__device__ inline void bias_sums(const BiasArgs& a, int wg, float* s_sum)
{
    const int m = min(wg * 64 + (int)threadIdx.x % 64, a.M - 1), w = threadIdx.x / 64;
    float v = 0.0f;
    for (int p0 = w; w < 4 && p0 < a.parts; p0 += 4 * 16) {
        float p[16];
#pragma unroll
        for (int i = 0; i < 16; ++i)
            p[i] = p0 + 4 * i < a.parts ? a.partial[(int64_t)(p0 + 4 * i) * a.M + m] : 0.0f;
#pragma unroll
        for (int i = 0; i < 16; ++i)
            v += p[i];
    }
    if (w < 4)
        s_sum[threadIdx.x] = v;
    __syncthreads();
    if (w == 0 && wg * 64 + (int)threadIdx.x < a.M)
        a.dbias[m] = (s_sum[threadIdx.x] + s_sum[64 + threadIdx.x]) + (s_sum[128 + threadIdx.x] + s_sum[192 + threadIdx.x]);
}

__global__ __launch_bounds__(256) void k_fused_bias(BiasArgs a)
{
    __shared__ float s_sum[256];
    bias_sums(a, blockIdx.x, s_sum);
}

// --- many rows -------------------------------------------------------------

// 16 bytes per lane from `off` of the resource (plus `at`) to LDS at `to` + 16 lane,
// without a register in between; past the resource: zeros.  The compiler does not
// see the write: the caller waits.
__device__ inline void load_to_lds(__amdgpu_buffer_rsrc_t rsrc, uint32_t off, uint32_t at, uint32_t to)
{
    asm volatile("s_mov_b32 m0, %2\n\tbuffer_load_dwordx4 %0, %1, %3 offen lds" ::"v"(off), "s"(rsrc),
                 "s"(__builtin_amdgcn_readfirstlane(to)), "s"(__builtin_amdgcn_readfirstlane(at))
                 : "memory");
}

// All but the wave's N newest loads have landed.
template <int N>
__device__ inline void wait_loads()
{
    asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory");
}

__device__ inline uint32_t lds_address(const void* p)
{
    return (uint32_t)(uintptr_t)(const __attribute__((address_space(3))) void*)p;
}

template <int NS, int MT, int NT, int WM, int WN>
constexpr int fused_stage_bytes() { return NS * 16 * NT * WN * 128 + WM * WN * MT * 1024; }

template <int NS, int MT, int NT, int WM, int WN, int D, int KS>
constexpr int fused_tile_lds()
{
    constexpr int rings = KS * D * fused_stage_bytes<NS, MT, NT, WM, WN>();
    constexpr int joining = (KS - 1) * WM * WN * MT * NT * 1024, turning = WM * WN * 2 * 16 * 16 * MT * 4;
    return rings > joining + turning ? rings : joining + turning;
}

// 16 MT WM outputs x 16 NT WN rows per workgroup of WM x WN waves.  The
// activations are NS planes of 16-bit parts (BF16 or F16 rows as they are, FP32
// ones and gradients in scaled F16 planes), rows of ld_x elements at 16-byte boundaries, n_in a
// multiple of 8.  Two planes may also lie side by side in a row (NS = 1): steps past
// w_steps, the second plane's, take the same weights again.  A ring of D stages in LDS holds 64 inputs of the rows and, for
// each wave, of its weights; a stage is fetched D - 1 steps ahead by loads that
// need no registers.  A row of a stage is 8 chunks of 16 bytes; chunk c of row r
// lies at c ^ (r % 8) (the lanes' global chunks are exchanged), so that an
// operand read's rows fall into different banks.  At the end each wave turns its
// sums around in LDS, 32 rows at a time, so that they leave as whole vectors of
// neighbouring outputs, past the caches, where they would only push the operands out
// (16,384 rows of 6144, BF16, and the values before the activation: 341 us through the
// caches, 321 past them; 2500 rows 52.7 and 51.4).
// KS groups of these waves share the steps, each with a ring of its own, and the first
// adds up their sums: where there are fewer tiles than compute units, one group leaves
// most of its unit's issue slots empty.
// Bound by how densely the waves issue products between their waits: 16,384 BF16 rows
// of 1536 -> 6144 with GELU and the values before it 319 us, 970 TFLOP/s (the product
// alone 264 us, 1174 TFLOP/s); 2500 FP32 rows, two planes, 91 us and 1034 TFLOP/s, the
// matrix units busy 45% of the time, LDS 4%; 8192 rows of 6144 -> 1536, two planes, 243 us
// and 1272 TFLOP/s, 59%.
// Codes widened by byte moves and packed F16 sums instead of conversions: no change.
template <typename OT, int NS, int MT, int NT, int WM, int WN, int D, int KS>
__global__ __launch_bounds__(64 * WM * WN * KS, KS == 1 ? 2 : KS) void k_fused_tile(FusedArgs a)
{
    constexpr int kThreads = 64 * WM * WN, kRows = 16 * NT * WN;  // threads of a group
    constexpr int kChunks = kRows * 8 / kThreads;  // 16-byte chunks of a plane that a thread fetches per step
    constexpr int kStage = fused_stage_bytes<NS, MT, NT, WM, WN>();
    constexpr int kLoads = NS * kChunks + MT;      // of a wave and step
    static_assert(kChunks >= 1 && kRows * 8 % kThreads == 0, "every thread fetches whole chunks");
    static_assert(NT % 2 == 0, "sums are turned around in pairs of row tiles");
    // From three stages on, the next step's is there one step early, and is read into
    // registers while this step's is multiplied.
    constexpr bool kEarly = D >= 3;
    constexpr int kBehind = kEarly ? (D - 3) * kLoads : 0;  // loads that may be on their way at a wait
    static_assert(kBehind < 64, "the load counter holds what is in flight");
    // With two stages, the next step's weights are needed half a step before its rows.  Asked
    // for first, they leave the rows the whole step (two planes, FP32 gradient of 2500 rows:
    // 139 us with both waited for half-way, 133 so; one plane, 16,384 rows: 334 and 341).
    constexpr bool kWeightsFirst = !kEarly && NS == 2;
    extern __shared__ u32x4 s_fused[];
    // Neighbouring workgroups of one XCD (every eighth) take tiles of a group
    // of 8 output tiles, so that they share both operands in its L2.
    const int plane_tiles = a.out_tiles * a.row_tiles, total = plane_tiles * a.splits, per_xcd = (total + 7) / 8;
    if (a.bias_sums.dbias && (int)blockIdx.x >= 8 * per_xcd)
        return bias_sums(a.bias_sums, blockIdx.x - 8 * per_xcd, reinterpret_cast<float*>(s_fused));
    const int place = (int)(blockIdx.x % 8) * per_xcd + blockIdx.x / 8;
    if ((int)(blockIdx.x / 8) >= per_xcd || place >= total)
        return;
    const int split = place / plane_tiles, id = place % plane_tiles;
    const int group = id / (8 * a.row_tiles), in_group = min(8, a.out_tiles - group * 8);
    const int out_tile = group * 8 + id % (8 * a.row_tiles) % in_group;
    const int row_tile = id % (8 * a.row_tiles) / in_group;
    const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
    const int team = KS == 1 ? 0 : wave / (WM * WN), w = KS == 1 ? wave : wave % (WM * WN);
    const int tid = KS == 1 ? (int)threadIdx.x : (int)threadIdx.x % kThreads;
    // every team walks `walk` steps; it has `steps` of them
    const int mine = min(a.split_steps, a.steps - split * a.split_steps), walk = (mine + KS - 1) / KS;
    const int first = min(split * a.split_steps + team * walk, a.steps - 1), steps = min(walk, mine - team * walk);
    const int g = lane / 16, c = lane % 16;
    const int wm = w % WM, wn = w / WM;
    const int tiles = (a.n_out + kFusedTile - 1) / kFusedTile;
    const int tile0 = (out_tile * WM + wm) * MT;
    const int64_t b0 = (int64_t)row_tile * kRows;

    const __amdgpu_buffer_rsrc_t wr = weight_resource(a.P, kBufMaxBytes);
    uint32_t w_at[MT];
#pragma unroll
    for (int t = 0; t < MT; ++t)  // tiles past the outputs repeat the last one; their results are not stored
        w_at[t] = (uint32_t)min(tile0 + t, tiles - 1) * a.w_steps * 1024u;
    __amdgpu_buffer_rsrc_t xr[NS];
#pragma unroll
    for (int p = 0; p < NS; ++p)
        xr[p] = rows_resource(static_cast<const uint16_t*>(a.x) + p * a.plane + b0 * a.ld_x);
    const int chunk = tid % 8 ^ tid / 8 % 8;
    uint32_t x_off[kChunks];  // bytes, of this thread's chunk of step 0
#pragma unroll
    for (int i = 0; i < kChunks; ++i) {
        const int64_t r = min((int64_t)(i * (kThreads / 8) + tid / 8), a.B - 1 - b0);
        x_off[i] = (uint32_t)(r * a.ld_x + first * kFusedStep + 8 * chunk) * 2u;
    }
    u32x4* const s_ring = s_fused + team * D * (kStage / 16);
    const uint32_t lds = lds_address(s_ring);
    constexpr int kWeights = NS * kRows * 128;  // of a stage: where the waves' weights begin
    // Step s of this workgroup's to stage `buf`; past the last, and past a row's end, zeros.
    auto fetch = [&](int buf, int s) __attribute__((always_inline)) {
        const bool live = s < steps && (first + s) * kFusedStep + 8 * chunk < a.n_in;
        const uint32_t at = s < steps ? s : 0, to = lds + buf * kStage;
        const uint32_t step = first + at, w_step = step - (step >= (uint32_t)a.w_steps ? a.w_steps : 0);
        auto weights = [&]() __attribute__((always_inline)) {
#pragma unroll
            for (int t = 0; t < MT; ++t)
                load_to_lds(wr, s < steps ? lane * 16u : kOutOfRange, w_at[t] + w_step * 1024u,
                            to + kWeights + (w * MT + t) * 1024);
        };
        if (kWeightsFirst)
            weights();
#pragma unroll
        for (int p = 0; p < NS; ++p)
#pragma unroll
            for (int i = 0; i < kChunks; ++i)
                load_to_lds(xr[p], live ? x_off[i] : kOutOfRange, at * 128u,
                            to + (p * kRows + i * (kThreads / 8) + w * 8) * 128);
        if (!kWeightsFirst)
            weights();
    };
    f32x4 acc[MT][NT];
#pragma unroll
    for (int t = 0; t < MT; ++t)
#pragma unroll
        for (int n = 0; n < NT; ++n)
            acc[t][n] = f32x4{};
    u32x4 wt[MT], wo[2][MT];  // a step's codes; the operands of its two halves
    const u32x4* const s_w = s_ring + kWeights / 16 + w * MT * 64 + lane;
#pragma unroll
    for (int s = 0; s < D - 1; ++s)
        fetch(s, s);
    wait_loads<kBehind>();
#pragma unroll
    for (int t = 0; t < MT; ++t) {
        wt[t] = s_w[t * 64];
        wo[0][t] = widen_codes<OT>(wt[t][0], wt[t][1]);
    }
    __syncthreads();
    // One step, in items of one operand of activations times MT of weights.  While an
    // item's products run, part of the next half's weights is widened and the
    // operand two items ahead is read.  A wave issues in order, so only work between
    // two products runs beside them: the order is pinned.
    constexpr int kHalf = NT * NS, kItems = 2 * kHalf;
    // (waves that multiply go before the waves of another workgroup that store)
    __builtin_amdgcn_s_setprio(1);
    int cur = 0;
    const int c0 = g ^ (c % 8), c1 = (4 + g) ^ (c % 8);
    auto read = [&](int stage, int item) __attribute__((always_inline)) {
        const int h = item / kHalf, n = item % kHalf / NS, p = item % NS;
        return s_ring[stage * (kStage / 16) + ((p * kRows + (wn * NT + n) * 16 + c) * 8 + (h == 0 ? c0 : c1))];
    };
    if constexpr (kEarly) {
        // all of the next step's operands and codes are read while this step's are multiplied
        u32x4 xs[2][kItems], ws[2][MT];
#pragma unroll
        for (int item = 0; item < kItems; ++item)
            xs[0][item] = read(0, item);
#pragma unroll
        for (int t = 0; t < MT; ++t)
            ws[0][t] = wt[t];
        auto step = [&](auto parity, int s) __attribute__((always_inline)) {
            constexpr int q = decltype(parity)::value;
            const int next = cur + 1 == D ? 0 : cur + 1, last = cur == 0 ? D - 1 : cur - 1;
#pragma unroll
            for (int t = 0; t < MT; ++t)
                ws[1 - q][t] = s_w[next * (kStage / 16) + t * 64];
#pragma unroll
            for (int item = 0; item < kItems; ++item)
                xs[1 - q][item] = read(next, item);
            fetch(last, s + D - 1);
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int item = 0; item < kItems; ++item) {
                const int h = item / kHalf, in_half = item % kHalf;
#pragma unroll
                for (int t = 0; t < MT; ++t) {
                    acc[t][in_half / NS] = mfma16<OT>(wo[h][t], xs[q][item], acc[t][in_half / NS]);
#pragma unroll
                    for (int v = 0; v < 4 * MT; ++v)
                        if (v * kHalf / 4 == in_half * MT + t)
                            wo[1 - h][v / 4][v % 4] = widen_pair<OT>(h == 0 ? ws[q][v / 4][2 + v % 4 / 2] : ws[1 - q][v / 4][v % 4 / 2], v % 2);
                    __builtin_amdgcn_sched_barrier(0);
                }
            }
            cur = next;
            wait_loads<kBehind>();
            __syncthreads();
        };
        for (int s = 0; s < walk; s += 2) {  // (a step past the last multiplies zeros)
            step(std::integral_constant<int, 0>{}, s);
            step(std::integral_constant<int, 1>{}, s + 1);
        }
    } else {
        for (int s = 0; s < walk; ++s) {
            const int next = cur + 1 == D ? 0 : cur + 1, last = cur == 0 ? D - 1 : cur - 1;
            u32x4 xo[3];
            xo[0] = read(cur, 0);
            xo[1] = read(cur, 1);
            fetch(last, s + D - 1);
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int item = 0; item < kItems; ++item) {
                const int h = item / kHalf, in_half = item % kHalf;
                if (item + 2 < kItems)
                    xo[(item + 2) % 3] = read(cur, item + 2);
                if (item == kHalf) {
                    // this wave's weights of the next step are there; they are its own
                    wait_loads<kWeightsFirst ? NS * kChunks : 0>();
#pragma unroll
                    for (int t = 0; t < MT; ++t)
                        wt[t] = s_w[next * (kStage / 16) + t * 64];
                }
#pragma unroll
                for (int t = 0; t < MT; ++t) {
                    acc[t][in_half / NS] = mfma16<OT>(wo[h][t], xo[item % 3], acc[t][in_half / NS]);
                    // a share of the 4 MT registers of the next half (of the next step, one item late: its codes are on their way)
#pragma unroll
                    for (int v = 0; v < 4 * MT; ++v) {
                        const int slot = h == 0 ? v * kHalf / 4 : MT + v * (kHalf - 1) / 4;
                        if (slot == in_half * MT + t)
                            wo[1 - h][v / 4][v % 4] = widen_pair<OT>(wt[v / 4][(h == 0 ? 2 : 0) + v % 4 / 2], v % 2);
                    }
                    __builtin_amdgcn_sched_barrier(0);
                }
            }
            cur = next;
            if (kWeightsFirst)
                wait_loads<0>();
            __syncthreads();
        }
    }
    __builtin_amdgcn_s_setprio(0);
    // the zeros fetched past the last step have landed everywhere before LDS is used anew
    wait_loads<0>();
    __syncthreads();
    if constexpr (KS > 1) {
        f32x4* const s_join = reinterpret_cast<f32x4*>(s_fused) + (w * MT * NT) * 64 + lane;
        constexpr int kTeam = WM * WN * MT * NT * 64;
        if (team > 0) {
#pragma unroll
            for (int t = 0; t < MT; ++t)
#pragma unroll
                for (int n = 0; n < NT; ++n)
                    s_join[(team - 1) * kTeam + (t * NT + n) * 64] = acc[t][n];
        }
        __syncthreads();
        if (team > 0)
            return;
#pragma unroll
        for (int k = 0; k < KS - 1; ++k)
#pragma unroll
            for (int t = 0; t < MT; ++t)
#pragma unroll
                for (int n = 0; n < NT; ++n)
                    acc[t][n] += s_join[k * kTeam + (t * NT + n) * 64];
    }
    float undo[NT];  // a lane's results belong to one row of each tile
    if constexpr (__is_same(OT, f16)) {
#pragma unroll
        for (int n = 0; n < NT; ++n)
            undo[n] = a.row_scale ? a.row_scale[min(b0 + (wn * NT + n) * 16 + c, (int64_t)a.B - 1)] : 1.0f;
    }
    // 32 rows x 16 MT outputs at a time, in this wave's own part of LDS; the
    // 16-byte chunk q of row r lies at q ^ (r % (4 MT))
    // (behind the other teams' sums)
    f32x4* const s_out = reinterpret_cast<f32x4*>(s_fused) + (KS - 1) * WM * WN * MT * NT * 64 + w * 2 * 16 * 4 * MT;
    constexpr int kVecs = 2 * MT;  // of 8 outputs, in a row
    static_assert(64 % kVecs == 0, "a lane keeps its outputs");
    const int q = lane % kVecs * 2;
    OutputColumns<8> columns;
    columns.load(a, tile0 * 16 + 4 * q);
    const int64_t y_at = split * a.split_stride;
#pragma unroll
    for (int n0 = 0; n0 < NT; n0 += 2) {
#pragma unroll
        for (int n = 0; n < 2; ++n)
#pragma unroll
            for (int t = 0; t < MT; ++t)
                s_out[(n * 16 + c) * 4 * MT + ((4 * t + g) ^ (c % (4 * MT)))] =
                    __is_same(OT, f16) ? acc[t][n0 + n] * undo[n0 + n] : acc[t][n0 + n];
        __builtin_amdgcn_wave_barrier();
#pragma unroll 1
        for (int r = lane / kVecs; r < 32; r += 64 / kVecs) {
            const f32x4 lo = s_out[r * 4 * MT + (q ^ (r % 16 % (4 * MT)))];
            const f32x4 hi = s_out[r * 4 * MT + ((q + 1) ^ (r % 16 % (4 * MT)))];
            float z[8] = {lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
            columns.template store<true>(a, b0 + (wn * NT + n0) * 16 + r, z, y_at);
        }
        __builtin_amdgcn_wave_barrier();
    }
}

// The join, and the copy below, walk rows of vectors of 8: a wave along a row, the four waves
// of a workgroup on rows of their own.
inline dim3 row_grid(int64_t rows, int64_t vectors)
{
    const int64_t along = (vectors + 63) / 64, down = (rows + 3) / 4;
    return dim3((unsigned)along, (unsigned)(down < 65535 ? down : 65535));
}

// Joins the sums of a product whose steps were split, the parts in ascending order,
// then the epilogue.  part: [splits][B] rows of ld elements.  Bound by memory and its
// launch (four parts of 500 rows of 1536: 6.2 us for 15 MB).
__global__ __launch_bounds__(256) void k_fused_join(FusedArgs a, const float* __restrict__ part, int64_t ld)
{
    const int m = (blockIdx.x * 64 + threadIdx.x % 64) * 8;
    if (m >= ld)
        return;
    const int64_t stride = ld * a.B;
    OutputColumns<8> columns;
    columns.load(a, m);
    for (int64_t b = blockIdx.y * 4 + threadIdx.x / 64; b < a.B; b += gridDim.y * 4) {
        const float* p = part + b * ld + m;
        f32x8 sum = load8(p);
        for (int k = 1; k < a.splits; ++k)
            sum += load8(p + k * stride);
        const float undo = a.row_scale ? a.row_scale[b] : 1.0f;
        float z[8];
#pragma unroll
        for (int e = 0; e < 8; ++e)
            z[e] = sum[e] * undo;
        columns.store(a, b, z);
    }
}

// Copies rows of n 16-bit elements at any alignment for the product: rows of `ld`
// (n rounded up to 8) elements, zeros past n.  Bound by memory (2500 rows of 1536 of
// them, one element off: 7.6 us, 2.0 TB/s: 2-byte loads).
__global__ __launch_bounds__(256) void k_fused_align(const uint16_t* __restrict__ x, int64_t ld_x, int B, int n, int64_t ld,
                                                     uint16_t* __restrict__ out)
{
    const int k = (blockIdx.x * 64 + threadIdx.x % 64) * 8;
    if (k >= ld)
        return;
    for (int64_t b = blockIdx.y * 4 + threadIdx.x / 64; b < B; b += gridDim.y * 4) {
        const uint16_t* h = x + b * ld_x + k;
        uint32_t r[4];
#pragma unroll
        for (int e = 0; e < 4; ++e)
            r[e] = (k + 2 * e < n ? h[2 * e] : 0u) | (k + 2 * e + 1 < n ? (uint32_t)h[2 * e + 1] << 16 : 0u);
        *reinterpret_cast<u32x4*>(out + b * ld + k) = u32x4{r[0], r[1], r[2], r[3]};
    }
}

// Cuts FP32 rows of n elements into two scaled F16 planes for the product.  Two
// roundings to 11 bits keep an element to 2^-23 of itself (one bit less than FP32
// holds; the sums' own rounding, 2^-24 of a partial sum per step, is larger) down to
// 2^-17 of the row's largest, and smaller ones to 2^-39 of that (F16's smallest step is
// 2^-24, the largest is scaled to 2^14 or more).  Three BF16 planes
// would keep every bit at any range, for half as much again in the product
// (1536 -> 6144, 2500 rows: 126 us, against 98; 500 rows 40 and 30).  The planes' rows
// have `ld` (n rounded up to 8) elements, zeros past n.  A workgroup walks a row, whose
// first 2,048 elements stay in registers between the two passes; bound by memory
// (2500 rows of 1536: 7.7 us, 4.0 TB/s read and written).
__global__ __launch_bounds__(256) void k_fused_cut(const float* __restrict__ x, int64_t ld_x, int B, int n, int64_t ld,
                                                   int64_t plane, uint16_t* __restrict__ out, float* __restrict__ undo, int vec)
{
    __shared__ float s_top[2][16];
    int turn = 0;
    for (int64_t b = blockIdx.x; b < B; b += gridDim.x, turn ^= 1) {
        const float* p = x + b * ld_x;
        const int k0 = threadIdx.x * 8;
        float held[8] = {};
        if (k0 < n)
            read_w<float, 8>(p + k0, held, vec && k0 + 8 <= n, n - k0);
        float top = largest(held, 0.0f);
        for (int k = k0 + 2048; k < n; k += 2048) {
            float v[8];
            read_w<float, 8>(p + k, v, vec && k + 8 <= n, n - k);
            top = largest(v, top);
        }
        const RowPower power = row_power(largest_of_waves(top, s_top[turn], 0, blockDim.x / 64));
        if (threadIdx.x == 0)
            undo[b] = power.undo;
        for (int k = k0; k < ld; k += 2048) {
            if (k > k0)
                read_w<float, 8>(p + k, held, vec && k + 8 <= n, n - k);
            put_planes(out + b * ld + k, plane, held, power.factor);
        }
    }
}

// --- gradient --------------------------------------------------------------

// g = dy act'(z) of 8 outputs, as they were loaded and then as they are.
template <typename T>
struct GateRaw {
    typename Vec8<T>::type dy, z;
};

// (VEC: rows of whole vectors at 16-byte boundaries, up to the last one)
template <typename T, bool VEC>
__device__ inline typename Vec8<T>::type gate_load(const T* p, int n)
{
    typename Vec8<T>::type v = (T)0.0f;
    if (VEC && n >= 8) {
        v = *reinterpret_cast<const typename Vec8<T>::type*>(p);
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (e < n)
                v[e] = p[e];
    }
    return v;
}

template <typename T, bool VEC>
__device__ inline GateRaw<T> gate_read(const T* dy, const T* pre, int m, int M, int act)
{
    GateRaw<T> r;
    r.dy = gate_load<T, VEC>(dy + m, M - m);
    r.z = act ? gate_load<T, VEC>(pre + m, M - m) : (typename Vec8<T>::type)(T)0.0f;
    return r;
}

template <typename T>
__device__ inline void gate_values(const GateRaw<T>& r, int act, float (&g)[8])
{
    float slope[8];
#pragma unroll
    for (int e = 0; e < 8; ++e)
        slope[e] = (float)r.z[e];
    act_slopes<8>(slope, act);
#pragma unroll
    for (int e = 0; e < 8; ++e)
        g[e] = (float)r.dy[e] * slope[e];
}

struct GateArgs {
    const void *dy, *pre;
    int64_t ld_dy, ld_pre;
    int act, B, M, rows;  // rows of a workgroup
    int along, groups;    // k_fused_gate: threads of a row, and the rows that a workgroup has at a time
    const float* scale;   // [M rounded up to 16]
    void* gs;             // NULL: only the bias gradient
    int width;            // elements that a row of gs has in a plane: M and zeros
    int64_t ld_gs, plane; // elements between rows and planes of gs
    float* undo;          // [B] inverses of the rows' scalings
    float* partial;       // [workgroups down][M] column sums of g, or NULL
};

// Rows of up to 8,192 outputs in whole vectors: a workgroup walks `rows` of them, `groups`
// at a time, g * scale of a row staying in registers until the row's largest is known, and
// goes to gs in two scaled F16 planes (PLANES; else as FP32 rows): g * scale is an FP32
// value whatever the type of dy, and dx may be FP32 (one plane, 11 bits, left 2e-4 of its
// size there).  A thread has one vector of outputs and their sums over the rows, which the groups join in LDS and leave in
// partial[workgroup]; the next row's loads are on their way while this one's largest is
// found.  Bound by memory, and about as much by the slope's arithmetic (8192 rows of
// 6144, BF16, 403 MB: 87 us, 4.6 TB/s).
constexpr int kGateParts = 512;  // the most parts that the bias gradient comes in

template <bool PLANES>
__device__ inline void gate_put(const GateArgs& a, int64_t b, int m, const float (&v)[8], float factor)
{
    if constexpr (PLANES)
        put_planes(static_cast<uint16_t*>(a.gs) + b * a.ld_gs + m, a.plane, v, factor);
    else
        write_w<float, 8>(static_cast<float*>(a.gs) + b * a.ld_gs + m, v, true, 8);
}

template <typename T, bool PLANES>
__global__ __launch_bounds__(1024) void k_fused_gate(GateArgs a)
{
    __shared__ float s_top[2][16];
    extern __shared__ u32x4 s_fused[];
    const int group = __builtin_amdgcn_readfirstlane((int)threadIdx.x / a.along), waves = a.along / 64;
    const int m0 = ((int)threadIdx.x - group * a.along) * 8;
    const int64_t b0 = (int64_t)blockIdx.x * a.rows, b1 = min((int64_t)a.B, b0 + a.rows);
    const T* const dy = static_cast<const T*>(a.dy);
    const T* const pre = static_cast<const T*>(a.pre);
    float sc[8], sum[8] = {};
    GateRaw<T> raw{};
    // (rows past the last are zeros)
    auto read = [&](int64_t b) __attribute__((always_inline)) {
        raw = gate_read<T, true>(dy + b * a.ld_dy, pre + b * a.ld_pre, m0, b < b1 ? a.M : 0, a.act);
    };
    read(b0 + group);
#pragma unroll
    for (int e = 0; e < 8; ++e)
        sc[e] = m0 + e < a.M ? a.scale[m0 + e] : 0.0f;
    int turn = 0;
    for (int64_t first = b0; first < b1; first += a.groups, turn ^= 1) {
        const int64_t b = first + group;
        const bool live = b < b1;
        float g[8];
        gate_values(raw, a.act, g);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            sum[e] += g[e];
            g[e] *= sc[e];
        }
        if (first + a.groups < b1)
            read(b + a.groups);
        if (!a.gs)
            continue;
        RowPower power{};
        if constexpr (PLANES) {
            power = row_power(largest_of_waves(largest(g, 0.0f), s_top[turn], group * waves, waves));
            if (live && m0 == 0)
                a.undo[b] = power.undo;
        }
        if (live && m0 < a.width)
            gate_put<PLANES>(a, b, m0, g, power.factor);
    }
    if (!a.partial)
        return;
    // [2 halves of a vector][groups - 1][along]
    f32x4* const s_sum = reinterpret_cast<f32x4*>(s_fused) + (int)threadIdx.x - a.along;
    const int total = (a.groups - 1) * a.along;
    if (group > 0) {
        s_sum[0] = f32x4{sum[0], sum[1], sum[2], sum[3]};
        s_sum[total] = f32x4{sum[4], sum[5], sum[6], sum[7]};
    }
    __syncthreads();
    if (group > 0)
        return;
    for (int k = 1; k < a.groups; ++k)
#pragma unroll
        for (int e = 0; e < 8; ++e)
            sum[e] += s_sum[k * a.along + e / 4 * total][e % 4];
    write_w<float, 8>(a.partial + blockIdx.x * (int64_t)a.M + m0, sum, a.M % 8 == 0 && m0 < a.M, a.M - m0);
}

// Any rows, in two kernels that each read dy and pre: the rows' largest, a workgroup a
// row; then a workgroup takes 256 outputs of `rows` rows.  Bound by memory (2500 FP32 rows
// of 12,000: 85 us for the 240 MB, and some 75 to read them again and write 120; one
// workgroup walking whole rows twice took 248 us, one that kept four vectors a thread
// ran out of registers and took 316).
template <typename T, bool VEC>
__global__ __launch_bounds__(512) void k_fused_gate_top(GateArgs a)
{
    __shared__ float s_top[16];
    const int64_t b = blockIdx.x;
    float top = 0.0f;
    for (int m = threadIdx.x * 8; m < a.M; m += 512 * 8) {
        float g[8];
        gate_values(gate_read<T, VEC>(static_cast<const T*>(a.dy) + b * a.ld_dy, static_cast<const T*>(a.pre) + b * a.ld_pre, m,
                                      a.M, a.act), a.act, g);
#pragma unroll
        for (int e = 0; e < 8; ++e)
            g[e] *= a.scale[min(m + e, a.M - 1)];
        top = largest(g, top);
    }
    top = largest_of_waves(top, s_top, 0, 8);
    if (threadIdx.x == 0)
        a.undo[b] = row_power(top).undo;
}

constexpr int kGateCols = 256;

template <typename T, bool PLANES, bool VEC>
__global__ __launch_bounds__(256) void k_fused_gate_columns(GateArgs a)
{
    const int m = blockIdx.x * kGateCols + threadIdx.x % 32 * 8;
    const int64_t b0 = (int64_t)blockIdx.y * a.rows, b1 = min((int64_t)a.B, b0 + a.rows);
    float sc[8], sum[8] = {};
#pragma unroll
    for (int e = 0; e < 8; ++e)
        sc[e] = m + e < a.M ? a.scale[m + e] : 0.0f;
    if (m < a.width)  // (g past M is 0)
        for (int64_t b = b0 + threadIdx.x / 32; b < b1; b += 8) {
            float g[8];
            gate_values(gate_read<T, VEC>(static_cast<const T*>(a.dy) + b * a.ld_dy, static_cast<const T*>(a.pre) + b * a.ld_pre,
                                          m, a.M, a.act), a.act, g);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                sum[e] += g[e];
                g[e] *= sc[e];
            }
            // (the power is the inverse of its inverse: 254 less its exponent)
            if (a.gs)
                gate_put<PLANES>(a, b, m, g, PLANES ? __uint_as_float((254u << 23) - __float_as_uint(a.undo[b])) : 1.0f);
        }
    if (!a.partial)
        return;
    __shared__ float s_sum[8][kGateCols];
#pragma unroll
    for (int e = 0; e < 8; ++e)
        s_sum[threadIdx.x / 32][threadIdx.x % 32 * 8 + e] = sum[e];
    __syncthreads();
    const int col = blockIdx.x * kGateCols + threadIdx.x;
    if (col < a.M) {
        float v = s_sum[0][threadIdx.x];
#pragma unroll
        for (int r = 1; r < 8; ++r)
            v += s_sum[r][threadIdx.x];
        a.partial[(int64_t)blockIdx.y * a.M + col] = v;
    }
}

}  // namespace spk
