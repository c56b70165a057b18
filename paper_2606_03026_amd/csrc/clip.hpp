// Norm of a list of gradients and its clipping (C ABI in include/spike_clip.h).
//
// The tensors are cut into chunks; a table of them lies in device memory.  The first
// kernel leaves one sum of squares per workgroup, the second adds these up in
// every workgroup alike and scales the chunks.  Bound by memory, the gradients being read twice (88 million FP32 elements: 205 us
// for 1.06 GB; with one vector on its way a thread 9% more; BF16 83).  Tensors off 16-byte boundaries go element by element (331
// and 217 in the same graph where aligned ones take 190 and 83).
#pragma once

#include "types.hpp"

namespace spk {

constexpr int kClipChunk = 16384;  // elements
constexpr int kClipFlight = 4;     // vectors of 8 that a thread has on their way
constexpr int kClipWgs = 2048;     // the most workgroups: each one's sum is read by all of the second kernel

struct ClipChunk {
    const void* in;
    void* out;
    int32_t n, type;
};

struct ClipArgs {
    const ClipChunk* chunks;
    int64_t n;
    double* partial;
    int wgs;  // of both kernels
    float max_norm;
    float* result;
};

// Sum over the workgroup, the same in every thread; s: 4 doubles of LDS.
__device__ inline double clip_sum(double v, double* s)
{
#pragma unroll
    for (int d = 32; d > 0; d /= 2)
        v += __shfl_xor(v, d);
    if (threadIdx.x % 64 == 0)
        s[threadIdx.x / 64] = v;
    __syncthreads();
    v = (s[0] + s[1]) + (s[2] + s[3]);
    __syncthreads();
    return v;
}

template <typename T>
__device__ inline void clip_squares(const ClipChunk& c, double (&sum)[2])
{
    const T* const p = static_cast<const T*>(c.in);
    const int whole = ((uintptr_t)p & 15) == 0 ? c.n / 8 : 0;
    int i = threadIdx.x;
    for (; i + 256 * (kClipFlight - 1) < whole; i += 256 * kClipFlight) {
        typename Vec8<T>::type v[kClipFlight];
#pragma unroll
        for (int u = 0; u < kClipFlight; ++u)
            v[u] = *reinterpret_cast<const typename Vec8<T>::type*>(p + 8 * (i + 256 * u));
#pragma unroll
        for (int u = 0; u < kClipFlight; ++u)
#pragma unroll
            for (int e = 0; e < 8; ++e)
                sum[e % 2] = __builtin_fma((double)(float)v[u][e], (double)(float)v[u][e], sum[e % 2]);
    }
    for (; i < whole; i += 256) {
        const f32x8 v = load8(p + 8 * i);
#pragma unroll
        for (int e = 0; e < 8; ++e)
            sum[e % 2] = __builtin_fma((double)v[e], (double)v[e], sum[e % 2]);
    }
    for (i = whole * 8 + threadIdx.x; i < c.n; i += 256) {
        const double v = (double)(float)p[i];
        sum[0] = __builtin_fma(v, v, sum[0]);
    }
}

__global__ __launch_bounds__(256) void k_clip_squares(ClipArgs a)
{
    __shared__ double s_sum[4];
    double sum[2] = {0.0, 0.0};
    for (int64_t i = blockIdx.x; i < a.n; i += gridDim.x) {
        const ClipChunk c = a.chunks[i];
        switch (c.type) {
        case SPIKE_TYPE_F32: clip_squares<float>(c, sum); break;
        case SPIKE_TYPE_BF16: clip_squares<bf16>(c, sum); break;
        default: clip_squares<f16>(c, sum);
        }
    }
    const double all = clip_sum(sum[0] + sum[1], s_sum);
    if (threadIdx.x == 0)
        a.partial[blockIdx.x] = all;
}

template <typename T>
__device__ inline void clip_scale(const ClipChunk& c, float factor)
{
    const T* const p = static_cast<const T*>(c.in);
    T* const q = static_cast<T*>(c.out);
    const int whole = (((uintptr_t)p | (uintptr_t)q) & 15) == 0 ? c.n / 8 : 0;
    int i = threadIdx.x;
    for (; i + 256 * (kClipFlight - 1) < whole; i += 256 * kClipFlight) {
        f32x8 v[kClipFlight];
#pragma unroll
        for (int u = 0; u < kClipFlight; ++u)
            v[u] = load8(p + 8 * (i + 256 * u));
#pragma unroll
        for (int u = 0; u < kClipFlight; ++u)
            store8<T, true>(q + 8 * (i + 256 * u), v[u] * factor);
    }
    for (; i < whole; i += 256)
        store8(q + 8 * i, load8(p + 8 * i) * factor);
    for (i = whole * 8 + threadIdx.x; i < c.n; i += 256)
        q[i] = (T)in_fp32<T>((float)p[i] * factor);
}

__global__ __launch_bounds__(256) void k_clip_scale(ClipArgs a)
{
    __shared__ double s_sum[4];
    double sum = 0.0;
    for (int i = threadIdx.x; i < a.wgs; i += 256)
        sum += a.partial[i];
    const double norm = __builtin_sqrt(clip_sum(sum, s_sum));
    // (an infinite norm leaves max / norm = 0, a NaN neither above nor below)
    const bool clip = norm > (double)a.max_norm && !__builtin_isinf(norm);
    const float factor = clip ? (float)((double)a.max_norm / norm) : 1.0f;
    if (blockIdx.x == 0 && threadIdx.x == 0) {
        a.result[0] = (float)norm;
        a.result[1] = factor;
    }
    // from the end: what the first kernel read last is still near
    for (int64_t i = a.n - 1 - blockIdx.x; i >= 0; i -= gridDim.x) {
        const ClipChunk c = a.chunks[i];
        if (c.in == c.out && !clip)
            continue;
        switch (c.type) {
        case SPIKE_TYPE_F32: clip_scale<float>(c, factor); break;
        case SPIKE_TYPE_BF16: clip_scale<bf16>(c, factor); break;
        default: clip_scale<f16>(c, factor);
        }
    }
}

}  // namespace spk
