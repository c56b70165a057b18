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

#include "types.hpp"

namespace spk {

constexpr int kFusedTile = 16;  // outputs and rows of one matrix instruction
constexpr int kFusedStep = 64;  // inputs of one weight load

inline int64_t fused_pad(int64_t n, int64_t to) { return (n + to - 1) / to * to; }
inline int64_t fused_packed_bytes(int64_t n_out, int64_t n_in)
{
    return fused_pad(n_out, kFusedTile) * fused_pad(n_in, kFusedStep);
}

// Lays out Q [M][K] with its rows as outputs, or (TRANSPOSE) its columns.
template <bool TRANSPOSE>
__global__ __launch_bounds__(256) void k_fused_pack(const int8_t* __restrict__ Q, int K, int M, int8_t* __restrict__ P,
                                                    int64_t chunks)
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
    for (int j = 0; j < 16; ++j) {
        const int64_t k = k0 + j % 8 + j / 8 * 32;
        w.b[j] = o < n_out && k < n_in ? (TRANSPOSE ? Q[k * K + o] : Q[o * K + k]) : 0;
    }
    reinterpret_cast<u32x4*>(P)[i] = w.v;
}

// --- values ----------------------------------------------------------------

// Operand types of the matrix instructions: activations in BF16 parts, or F16 as they are.
template <typename XT> struct Operand { typedef bf16 type; };
template <> struct Operand<f16> { typedef f16 type; };

__device__ inline uint32_t high_halves(float lo, float hi)
{
    return __builtin_amdgcn_perm(__float_as_uint(hi), __float_as_uint(lo), 0x07060302u);
}

// 8 codes -> 8 operand values, exactly (a float holding one has its lower half zero).
template <typename OT>
__device__ inline u32x4 widen_codes(uint32_t w0, uint32_t w1)
{
    u32x4 r;
    for (int i = 0; i < 4; ++i) {
        const uint32_t w = i < 2 ? w0 : w1;
        const float a = (float)(int8_t)(w >> (i % 2 * 16)), b = (float)(int8_t)(w >> (i % 2 * 16 + 8));
        if constexpr (sizeof(OT) == 2 && __is_same(OT, f16)) {
            typedef __fp16 h2 __attribute__((ext_vector_type(2)));
            const h2 p = __builtin_amdgcn_cvt_pkrtz(a, b);
            r[i] = __builtin_bit_cast(uint32_t, p);
        } else {
            r[i] = high_halves(a, b);
        }
    }
    return r;
}

// What of x is left after its upper 16 bits are taken off as a BF16 part; nothing of an infinity.
__device__ inline float below_bf16(float x)
{
    const float r = x - __uint_as_float(__float_as_uint(x) & 0xffff0000u);
    return __builtin_isinf(x) ? 0.0f : r;
}

// 8 activations as they were loaded.
template <typename XT> struct Raw { u32x4 v; };
template <> struct Raw<float> { f32x4 v[2]; };

// Activations k .. k + 7 of a row that has n; zeros past it.
template <typename XT, bool VECX>
__device__ inline Raw<XT> load_raw(const XT* row, int k, int n)
{
    Raw<XT> r;
    if constexpr (sizeof(XT) == 4) {
        if (VECX && k + 8 <= n) {
            r.v[0] = *reinterpret_cast<const f32x4*>(row + k);
            r.v[1] = *reinterpret_cast<const f32x4*>(row + k + 4);
        } else {
            for (int e = 0; e < 8; ++e)
                r.v[e / 4][e % 4] = k + e < n ? row[k + e] : 0.0f;
        }
    } else {
        if (VECX && k + 8 <= n) {
            r.v = *reinterpret_cast<const u32x4*>(row + k);
        } else {
            const uint16_t* p = reinterpret_cast<const uint16_t*>(row);
            for (int e = 0; e < 4; ++e)
                r.v[e] = (k + 2 * e < n ? p[k + 2 * e] : 0u) | (k + 2 * e + 1 < n ? (uint32_t)p[k + 2 * e + 1] << 16 : 0u);
        }
    }
    return r;
}

// Their NS operand parts.
template <typename XT, int NS>
__device__ inline void split_raw(const Raw<XT>& r, u32x4 (&part)[NS])
{
    if constexpr (sizeof(XT) == 4) {
        for (int i = 0; i < 4; ++i) {
            float a = r.v[i / 2][i % 2 * 2], b = r.v[i / 2][i % 2 * 2 + 1];
            for (int s = 0; s < NS; ++s) {
                part[s][i] = high_halves(a, b);
                if (s + 1 < NS)
                    a = below_bf16(a), b = below_bf16(b);
            }
        }
    } else {
        part[0] = r.v;
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
// relative error 1.7e-7 over all a (least squares with weights raised where
// the error was largest, in double precision).
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

__device__ inline float act_value(float z, int act)
{
    switch (act) {
    case 1: return z > 0.0f ? z : z == z ? 0.0f : z;
    case 2: {
        const float tail = __builtin_amdgcn_exp2f(z * z * -0.72134752f) * gauss_tail(__builtin_fabsf(z));
        return z * (z < 0.0f ? tail : 1.0f - tail);
    }
    case 3: return z * __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(z * -1.44269504f));
    default: return z;
    }
}

__device__ inline float act_slope(float z, int act)
{
    switch (act) {
    case 1: return z > 0.0f ? 1.0f : z == z ? 0.0f : z;
    case 2: {
        const float e = __builtin_amdgcn_exp2f(z * z * -0.72134752f);
        const float tail = e * gauss_tail(__builtin_fabsf(z));
        return __builtin_fmaf(z, e * 0.39894228f, z < 0.0f ? tail : 1.0f - tail);
    }
    case 3: {
        const float s = __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(z * -1.44269504f));
        return s * __builtin_fmaf(z, 1.0f - s, 1.0f);
    }
    default: return 1.0f;
    }
}

// --- epilogue --------------------------------------------------------------

struct FusedArgs {
    const int8_t* P;     // weights, laid out
    int n_out, n_in, steps;
    const void* x;
    int64_t ld_x;
    int B;
    const float* scale;  // [n_out rounded up to 16], NULL: one
    const float* bias;
    int act;
    const void* residual;
    int64_t ld_residual;
    void* y;
    int y_type;
    int64_t ld_y;
    void* pre;
    int64_t ld_pre;
    int vec_out;         // rows of y, residual and pre go four elements at a time
    int out_tiles, row_tiles;
};

template <typename T>
__device__ inline f32x4 read4(const T* p, bool vec, int n)
{
    f32x4 v = {};
    if (vec) {
        typedef T t4 __attribute__((ext_vector_type(4)));
        v = __builtin_convertvector(*reinterpret_cast<const t4*>(p), f32x4);
    } else {
        for (int e = 0; e < 4; ++e)
            if (e < n)
                v[e] = (float)p[e];
    }
    return v;
}

template <typename T>
__device__ inline void write4(T* p, f32x4 v, bool vec, int n)
{
    for (int e = 0; e < 4; ++e)
        v[e] = in_fp32<T>(v[e]);
    if (vec) {
        typedef T t4 __attribute__((ext_vector_type(4)));
        *reinterpret_cast<t4*>(p) = __builtin_convertvector(v, t4);
    } else {
        for (int e = 0; e < 4; ++e)
            if (e < n)
                p[e] = (T)v[e];
    }
}

template <typename T>
__device__ inline void put_outputs(const FusedArgs& a, int m, int64_t b, f32x4 z, bool vec, int n)
{
    if (a.pre)
        write4(static_cast<T*>(a.pre) + b * a.ld_pre + m, z, vec, n);
    if (a.act)
        for (int e = 0; e < 4; ++e)
            z[e] = act_value(z[e], a.act);
    if (a.residual)
        z += read4(static_cast<const T*>(a.residual) + b * a.ld_residual + m, vec, n);
    write4(static_cast<T*>(a.y) + b * a.ld_y + m, z, vec, n);
}

// Outputs m .. m + 3 of row b from their sums; m is a multiple of 4.
__device__ inline void fused_store(const FusedArgs& a, int m, int b, f32x4 sum)
{
    if (b >= a.B || m >= a.n_out)
        return;
    const int n = min(4, a.n_out - m);
    const bool vec = a.vec_out && n == 4;
    f32x4 z = sum;
    if (a.scale)
        z *= *reinterpret_cast<const f32x4*>(a.scale + m);
    if (a.bias)
        for (int e = 0; e < 4; ++e)
            z[e] += e < n ? a.bias[m + e] : 0.0f;
    switch (a.y_type) {
    case SPIKE_TYPE_F32: return put_outputs<float>(a, m, b, z, vec, n);
    case SPIKE_TYPE_BF16: return put_outputs<bf16>(a, m, b, z, vec, n);
    default: return put_outputs<f16>(a, m, b, z, vec, n);
    }
}

// --- few rows --------------------------------------------------------------

// Up to 16 NB rows: a workgroup takes 16 MT outputs and all inputs, its WK
// waves sharing the 64-input steps; the waves' sums are joined in LDS.  Bound
// by the weights' bytes (and, at one tile of rows, by latency).  Rows that are
// not there cost no loads, only idle columns of the matrix instruction.
template <typename XT, int NS, int NB, int MT, int WK, bool VECX>
__global__ __launch_bounds__(64 * WK) void k_fused_rows(FusedArgs a)
{
    typedef typename Operand<XT>::type OT;
    constexpr int U = MT * NB >= 4 ? 1 : MT * NB >= 2 ? 2 : 4;  // steps in flight
    const int lane = threadIdx.x % 64, w = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
    const int g = lane / 16, c = lane % 16;
    const int tile0 = blockIdx.x * MT, b0 = blockIdx.y * 16 * NB;
    const int tiles = (a.n_out + kFusedTile - 1) / kFusedTile;
    f32x4 acc[MT][NB] = {};
    for (int s0 = w; s0 < a.steps; s0 += WK * U) {
        u32x4 wt[U][MT];
        Raw<XT> x[U][NB][2];
        for (int u = 0; u < U; ++u) {
            const int s = s0 + u * WK;
            const bool live = s < a.steps;
            for (int t = 0; t < MT; ++t) {
                wt[u][t] = u32x4{};
                if (live && tile0 + t < tiles)
                    wt[u][t] = *reinterpret_cast<const u32x4*>(a.P + (((int64_t)(tile0 + t) * a.steps + s) * 64 + lane) * 16);
            }
            for (int t = 0; t < NB; ++t)
                for (int h = 0; h < 2; ++h) {
                    x[u][t][h] = Raw<XT>{};
                    const int b = b0 + 16 * t + c;
                    if (live && b < a.B)
                        x[u][t][h] = load_raw<XT, VECX>(static_cast<const XT*>(a.x) + b * a.ld_x, s * kFusedStep + 32 * h + 8 * g,
                                                        a.n_in);
                }
        }
        for (int u = 0; u < U; ++u)
            for (int h = 0; h < 2; ++h) {
                u32x4 wo[MT];
                for (int t = 0; t < MT; ++t)
                    wo[t] = widen_codes<OT>(wt[u][t][2 * h], wt[u][t][2 * h + 1]);
                for (int n = 0; n < NB; ++n) {
                    u32x4 part[NS];
                    split_raw<XT, NS>(x[u][n][h], part);
                    for (int p = 0; p < NS; ++p)
                        for (int t = 0; t < MT; ++t)
                            acc[t][n] = mfma16<OT>(wo[t], part[p], acc[t][n]);
                }
            }
    }
    __shared__ f32x4 s_sum[WK > 1 ? WK : 1][MT * NB][64];
    for (int t = 0; t < MT; ++t)
        for (int n = 0; n < NB; ++n)
            s_sum[w][t * NB + n][lane] = acc[t][n];
    __syncthreads();
    for (int q = w; q < MT * NB; q += WK) {
        f32x4 sum = s_sum[0][q][lane];
        for (int v = 1; v < WK; ++v)
            sum += s_sum[v][q][lane];
        fused_store(a, (tile0 + q / NB) * 16 + 4 * g, b0 + q % NB * 16 + c, sum);
    }
}

// --- many rows -------------------------------------------------------------

// 16 MT WM outputs x 16 NT WN rows per workgroup of WM x WN waves.  Each step
// of 64 inputs: weights straight from their layout to registers, one step
// ahead; activations through registers to LDS, two steps ahead, their parts
// made on the way.  A row of the LDS tile is 8 chunks of 16 bytes; chunk c of
// row r lies at c ^ (r % 8), so that the 16 rows of an operand read fall into
// different banks.
template <typename XT, int NS, int MT, int NT, int WM, int WN, bool VECX>
__global__ __launch_bounds__(64 * WM * WN) void k_fused_tile(FusedArgs a)
{
    typedef typename Operand<XT>::type OT;
    constexpr int kThreads = 64 * WM * WN, kRows = 16 * NT * WN;
    constexpr int kChunks = kRows * 8 / kThreads;
    static_assert(kChunks >= 1 && kRows * 8 % kThreads == 0, "every thread stages whole chunks");
    __shared__ u32x4 s_x[2][NS][kRows * 8];
    // Neighbouring workgroups of one XCD (every eighth) take tiles of a group
    // of 8 output tiles, so that they share both operands in its L2.
    const int total = a.out_tiles * a.row_tiles, per_xcd = (total + 7) / 8;
    const int id = (int)(blockIdx.x % 8) * per_xcd + blockIdx.x / 8;
    if ((int)(blockIdx.x / 8) >= per_xcd || id >= total)
        return;
    const int group = id / (8 * a.row_tiles), in_group = min(8, a.out_tiles - group * 8);
    const int out_tile = group * 8 + id % (8 * a.row_tiles) % in_group;
    const int row_tile = id % (8 * a.row_tiles) / in_group;
    const int lane = threadIdx.x % 64, w = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
    const int g = lane / 16, c = lane % 16;
    const int wm = w % WM, wn = w / WM;
    const int tiles = (a.n_out + kFusedTile - 1) / kFusedTile;
    const int tile0 = (out_tile * WM + wm) * MT, b0 = row_tile * kRows;

    const u32x4* wp[MT];
    for (int t = 0; t < MT; ++t)  // tiles past the outputs repeat the last one; their results are not stored
        wp[t] = reinterpret_cast<const u32x4*>(a.P) + (int64_t)min(tile0 + t, tiles - 1) * a.steps * 64 + lane;
    const XT* xp[kChunks];
    for (int i = 0; i < kChunks; ++i) {
        const int r = i * (kThreads / 8) + threadIdx.x / 8;
        xp[i] = static_cast<const XT*>(a.x) + (int64_t)min(b0 + r, a.B - 1) * a.ld_x;
    }
    const int chunk = threadIdx.x % 8;
    u32x4 wt[MT];
    Raw<XT> raw[kChunks];
    auto load_w = [&](int s) {
        for (int t = 0; t < MT; ++t)
            wt[t] = wp[t][s * 64];
    };
    auto load_x = [&](int s) {
        for (int i = 0; i < kChunks; ++i)
            raw[i] = load_raw<XT, VECX>(xp[i], s * kFusedStep + 8 * chunk, a.n_in);
    };
    auto stage = [&](int buf) {
        for (int i = 0; i < kChunks; ++i) {
            const int r = i * (kThreads / 8) + threadIdx.x / 8;
            u32x4 part[NS];
            split_raw<XT, NS>(raw[i], part);
            for (int p = 0; p < NS; ++p)
                s_x[buf][p][r * 8 + (chunk ^ (r % 8))] = part[p];
        }
    };
    f32x4 acc[MT][NT] = {};
    load_x(0);
    load_w(0);
    stage(0);
    if (a.steps > 1)
        load_x(1);
    __syncthreads();
    for (int s = 0; s < a.steps; ++s) {
        u32x4 wo[2][MT];
        for (int h = 0; h < 2; ++h)
            for (int t = 0; t < MT; ++t)
                wo[h][t] = widen_codes<OT>(wt[t][2 * h], wt[t][2 * h + 1]);
        if (s + 1 < a.steps)
            load_w(s + 1);
        for (int h = 0; h < 2; ++h)
            for (int n = 0; n < NT; ++n)
                for (int p = 0; p < NS; ++p) {
                    const int r = (wn * NT + n) * 16 + c;
                    const u32x4 xo = s_x[s % 2][p][r * 8 + ((4 * h + g) ^ (r % 8))];
                    for (int t = 0; t < MT; ++t)
                        acc[t][n] = mfma16<OT>(wo[h][t], xo, acc[t][n]);
                }
        if (s + 1 < a.steps)
            stage((s + 1) % 2);
        if (s + 2 < a.steps)
            load_x(s + 2);
        __syncthreads();
    }
    for (int n = 0; n < NT; ++n)
        for (int t = 0; t < MT; ++t)
            fused_store(a, (tile0 + t) * 16 + 4 * g, b0 + (wn * NT + n) * 16 + c, acc[t][n]);
}

// --- gradient --------------------------------------------------------------

// g = dy act'(z): per workgroup 256 outputs and `rows` rows.  g * scale goes to
// gs (rows of ld_gs elements) for the product, and the column sums of g over
// these rows to partial[row block].  Bound by memory.
constexpr int kGateCols = 256;

template <typename T, typename TG, bool VEC>
__global__ __launch_bounds__(256) void k_fused_gate(const T* __restrict__ dy, int64_t ld_dy, const T* __restrict__ pre,
                                                    int64_t ld_pre, int act, int B, int M, int rows,
                                                    const float* __restrict__ scale, TG* __restrict__ gs, int64_t ld_gs,
                                                    float* __restrict__ partial)
{
    const int m = blockIdx.x * kGateCols + threadIdx.x % 32 * 8;
    const int64_t b0 = (int64_t)blockIdx.y * rows, b1 = min((int64_t)B, b0 + rows);
    const bool full = VEC && m + 8 <= M;
    float sc[8], sum[8] = {};
    for (int e = 0; e < 8; ++e)
        sc[e] = m + e < M ? scale[m + e] : 0.0f;
    if (m < M)
        for (int64_t b = b0 + threadIdx.x / 32; b < b1; b += 8) {
            f32x8 g = {}, z = {};
            if (full) {
                g = load8(dy + b * ld_dy + m);
                if (act)
                    z = load8(pre + b * ld_pre + m);
            } else {
                for (int e = 0; e < 8; ++e)
                    if (m + e < M) {
                        g[e] = (float)dy[b * ld_dy + m + e];
                        if (act)
                            z[e] = (float)pre[b * ld_pre + m + e];
                    }
            }
            f32x8 out;
            for (int e = 0; e < 8; ++e) {
                if (act)
                    g[e] *= act_slope(z[e], act);
                sum[e] += g[e];
                out[e] = g[e] * sc[e];
            }
            if (gs)
                store8(gs + b * ld_gs + m, out);  // rows of gs are padded to whole vectors
        }
    if (!partial)
        return;
    __shared__ float s_sum[8][kGateCols];
    for (int e = 0; e < 8; ++e)
        s_sum[threadIdx.x / 32][threadIdx.x % 32 * 8 + e] = sum[e];
    __syncthreads();
    const int col = blockIdx.x * kGateCols + threadIdx.x;
    if (col < M) {
        float v = s_sum[0][threadIdx.x];
        for (int r = 1; r < 8; ++r)
            v += s_sum[r][threadIdx.x];
        partial[(int64_t)blockIdx.y * M + col] = v;
    }
}

__global__ __launch_bounds__(64) void k_fused_bias(const float* __restrict__ partial, int parts, int M,
                                                   float* __restrict__ dbias)
{
    const int m = blockIdx.x * 64 + threadIdx.x;
    if (m >= M)
        return;
    float v = 0.0f;
    for (int p = 0; p < parts; ++p)
        v += partial[(int64_t)p * M + m];
    dbias[m] = v;
}

}  // namespace spk
