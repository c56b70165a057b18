// Penalties, biases and masks on logits (C ABI in include/head_logits.h).
#pragma once

#include "types.hpp"

namespace spk {

constexpr int kLogitsPart = 2048;  // tokens of a workgroup: 8 a thread

struct LogitsArgs {
    const void* logits;
    int64_t ld_logits;
    int S, n, V;
    const int32_t* ids;
    int64_t ld_ids;
    int L;
    const int32_t *n_ids, *n_prompt, *drafts;
    const float *repetition, *presence, *frequency;
    const int32_t* bias_ids;
    const float* bias;
    int n_bias;
    const uint32_t* mask;
    int64_t ld_mask;
    void* out;
    int64_t ld_out;
    int parts;  // of a row
    int vec_ids;
};

constexpr uint32_t kLogitsPrompt = 1u << 31;  // beside a count: the token is the prompt's

// A workgroup takes 2,048 tokens of the n rows of a sequence.  It counts in LDS which of them the
// history names (whole numbers, so the order of the atomics does not matter) and where the list of biases names them last, then
// walks the rows; before row j it counts draft j - 1.
// VEC: rows of logits and out start on 16-byte boundaries; a thread has 8 neighbouring tokens, else every 256th.
template <typename T, bool VEC>
__global__ __launch_bounds__(256) void k_logits(LogitsArgs a)
{
    __shared__ uint32_t s_count[kLogitsPart];
    __shared__ int32_t s_bias[kLogitsPart];  // 1 + entry of the list, 0: none
    const int64_t units = (int64_t)a.S * a.parts;
    for (int64_t unit = blockIdx.x; unit < units; unit += gridDim.x) {
        const int64_t s = unit / a.parts;
        const int v0 = (int)(unit % a.parts) * kLogitsPart;
        const uint32_t here = (uint32_t)min(kLogitsPart, a.V - v0);
        for (int i = threadIdx.x; i < kLogitsPart; i += 256)
            s_count[i] = 0, s_bias[i] = 0;
        __syncthreads();
        if (a.ids) {
            const int32_t* const ids = a.ids + s * a.ld_ids;
            const int end = a.n_ids ? min(max(a.n_ids[s], 0), a.L) : a.L;
            const int start = a.n_prompt ? min(max(a.n_prompt[s], 0), end) : 0;
            auto name = [&](int32_t id, int at) __attribute__((always_inline)) {
                const uint32_t v = (uint32_t)id - (uint32_t)v0;
                if (v < here && id >= 0) {
                    if (at < start)
                        atomicOr(&s_count[v], kLogitsPrompt);
                    else
                        atomicAdd(&s_count[v], 1u);
                }
            };
            const int whole = a.vec_ids ? end / 4 : 0;
#pragma unroll 4
            for (int i = threadIdx.x; i < whole; i += 256) {
                const i32x4 id = *reinterpret_cast<const i32x4*>(ids + 4 * i);
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    name(id[e], 4 * i + e);
            }
            for (int i = whole * 4 + threadIdx.x; i < end; i += 256)
                name(ids[i], i);
        }
        for (int i = threadIdx.x; i < a.n_bias; i += 256) {
            const int32_t id = a.bias_ids[s * a.n_bias + i];
            const uint32_t v = (uint32_t)id - (uint32_t)v0;
            if (v < here && id >= 0)
                atomicMax(&s_bias[v], i + 1);
        }
        const float repetition = a.repetition ? a.repetition[s] : 1.0f;
        const float presence = a.presence ? a.presence[s] : 0.0f, frequency = a.frequency ? a.frequency[s] : 0.0f;
        for (int j = 0; j < a.n; ++j) {
            if (j > 0 && a.drafts && threadIdx.x == 0) {
                const int32_t id = a.drafts[s * (a.n - 1) + j - 1];
                const uint32_t v = (uint32_t)id - (uint32_t)v0;
                if (v < here && id >= 0)
                    s_count[v] += 1;
            }
            __syncthreads();
            const int64_t row = s * a.n + j;
            const T* const p = static_cast<const T*>(a.logits) + row * a.ld_logits + v0;
            T* const q = static_cast<T*>(a.out) + row * a.ld_out + v0;
            const uint32_t* const mask = a.mask ? a.mask + row * a.ld_mask + v0 / 32 : nullptr;
            auto at = [](int e) { return VEC ? (int)threadIdx.x * 8 + e : e * 256 + (int)threadIdx.x; };
            float x[8];
            const bool whole = VEC && threadIdx.x * 8 + 8 <= here;
            if (whole) {
                const f32x8 r = load8(p + threadIdx.x * 8);
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    x[e] = r[e];
            } else {
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    x[e] = (uint32_t)at(e) < here ? (float)p[at(e)] : 0.0f;
            }
            uint32_t allowed = 0xffu;  // one bit an element
            if (mask) {
                if constexpr (VEC) {
                    allowed = threadIdx.x * 8 < here ? mask[threadIdx.x / 4] >> (threadIdx.x % 4 * 8) : 0u;
                } else {
                    allowed = 0;
#pragma unroll
                    for (int e = 0; e < 8; ++e)
                        if ((uint32_t)at(e) < here)
                            allowed |= (mask[at(e) / 32] >> (at(e) % 32) & 1u) << e;
                }
            }
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const uint32_t c = s_count[at(e)];
                if (c != 0) {
                    x[e] = x[e] > 0.0f ? x[e] / repetition : x[e] * repetition;
                    const uint32_t said = c & ~kLogitsPrompt;
                    if (said != 0) {
                        x[e] = x[e] - frequency * (float)said;
                        x[e] = x[e] - presence;
                    }
                }
                const int32_t b = s_bias[at(e)];
                if (b != 0)
                    x[e] = x[e] + a.bias[s * a.n_bias + b - 1];
                if (!(allowed >> e & 1u))
                    x[e] = -__builtin_inff();
            }
            if (whole) {
                store8(q + threadIdx.x * 8, f32x8{x[0], x[1], x[2], x[3], x[4], x[5], x[6], x[7]});
            } else {
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    if ((uint32_t)at(e) < here)
                        q[at(e)] = (T)in_fp32<T>(x[e]);
            }
            __syncthreads();
        }
    }
}

}  // namespace spk
