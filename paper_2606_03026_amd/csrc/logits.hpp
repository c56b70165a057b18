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

// Elements of a row as they were loaded: 8 neighbours, or every 256th.
template <typename T, bool VEC>
struct LogitsRaw {
    typename Vec8<T>::type v;
    uint32_t allowed;  // one bit an element

    __device__ inline void load(const LogitsArgs& a, int64_t row, int v0, uint32_t here)
    {
        const T* const p = static_cast<const T*>(a.logits) + row * a.ld_logits + v0;
        const uint32_t* const mask = a.mask ? a.mask + row * a.ld_mask + v0 / 32 : nullptr;
        const uint32_t t = threadIdx.x;
        allowed = 0xffu;
        if (VEC && t * 8 + 8 <= here) {
            v = __builtin_nontemporal_load(reinterpret_cast<const typename Vec8<T>::type*>(p + t * 8));
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const uint32_t at = VEC ? t * 8 + e : e * 256 + t;
                v[e] = at < here ? p[at] : (T)0.0f;
            }
        }
        if (mask) {
            if constexpr (VEC) {
                allowed = t * 8 < here ? mask[t / 4] >> (t % 4 * 8) : 0u;
            } else {
                allowed = 0;
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const uint32_t at = e * 256 + t;
                    if (at < here)
                        allowed |= (mask[at / 32] >> (at % 32) & 1u) << e;
                }
            }
        }
    }
};

// (A quotient by the inverse and the remainder is as fast, 64 sequences of 5 rows 42.6 us either way, but off where the
// remainder is subnormal or the product overflows.)
__device__ inline float penalized(float x, float r) { return x > 0.0f ? x / r : x * r; }

// A workgroup takes 2,048 tokens of the n rows of a sequence.  It counts in LDS which of them the
// history names (whole numbers, so the order of the atomics does not matter) and where the list of biases names them last; then a
// thread holds what its 8 tokens have in registers and walks the rows, counting draft j - 1 before row j, with the next row's
// loads on their way.  VEC: rows of logits and out start on 16-byte boundaries; a thread has 8 neighbouring
// tokens, else every 256th.  Bound by memory where rows are many (64 sequences of 5 rows of 57,344 FP32: 42 us, 3.5 TB/s; BF16 35; rows
// off 16-byte boundaries 57 and 43; 48 with the counts read and the drafts
// counted in LDS between the rows; fewer registers spill and take 53 to 69),
// by the chain of reads where they are few.
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
        // what the list's start names is asked for before how long it is is known, and the first row beside it
        const int32_t* const ids = a.ids + s * a.ld_ids;
        const int in_fours = a.ids && a.vec_ids ? a.L / 4 : 0;
        i32x4 id[4];
        auto fours = [&](int i0, int end) __attribute__((always_inline)) {
#pragma unroll
            for (int u = 0; u < 4; ++u)
                id[u] = i0 + 256 * u < end ? *reinterpret_cast<const i32x4*>(ids + 4 * (int64_t)(i0 + 256 * u)) : i32x4{-1, -1, -1, -1};
        };
        fours(threadIdx.x, in_fours);
        LogitsRaw<T, VEC> raw;
        raw.load(a, s * a.n, v0, here);
        const float repetition = a.repetition ? a.repetition[s] : 1.0f;
        const float presence = a.presence ? a.presence[s] : 0.0f, frequency = a.frequency ? a.frequency[s] : 0.0f;
        const int end = a.n_ids ? min(max(a.n_ids[s], 0), a.L) : a.L;
        const int start = a.n_prompt ? min(max(a.n_prompt[s], 0), end) : 0;
#pragma unroll
        for (int i = 0; i < kLogitsPart / 256 / 4; ++i) {
            reinterpret_cast<u32x4*>(s_count)[threadIdx.x + 256 * i] = u32x4{};
            reinterpret_cast<u32x4*>(s_bias)[threadIdx.x + 256 * i] = u32x4{};
        }
        __syncthreads();
        if (a.ids) {
            auto name = [&](int32_t id, int at) __attribute__((always_inline)) {
                const uint32_t v = (uint32_t)id - (uint32_t)v0;
                if (v < here && id >= 0 && at < end) {
                    if (at < start)
                        atomicOr(&s_count[v], kLogitsPrompt);
                    else
                        atomicAdd(&s_count[v], 1u);
                }
            };
            for (int i0 = threadIdx.x; 4 * i0 < min(end, 4 * in_fours); i0 += 256 * 4) {
                if (i0 >= 256 * 4)
                    fours(i0, in_fours);
#pragma unroll
                for (int u = 0; u < 4; ++u)
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        name(id[u][e], 4 * (i0 + 256 * u) + e);
            }
            for (int i = in_fours * 4 + threadIdx.x; i < end; i += 256)
                name(ids[i], i);
        }
        for (int i = threadIdx.x; i < a.n_bias; i += 256) {
            const int32_t id = a.bias_ids[s * a.n_bias + i];
            const uint32_t v = (uint32_t)id - (uint32_t)v0;
            if (v < here && id >= 0)
                atomicMax(&s_bias[v], i + 1);
        }
        __syncthreads();
        auto at = [](int e) { return VEC ? (int)threadIdx.x * 8 + e : e * 256 + (int)threadIdx.x; };
        uint32_t count[8], any = 0, biased = 0;
        float bias[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            count[e] = s_count[at(e)];
            any |= count[e];
            const int32_t b = s_bias[at(e)];
            bias[e] = 0.0f;
            if (b != 0)
                bias[e] = a.bias[s * a.n_bias + b - 1], biased |= 1u << e;
        }
        for (int j = 0; j < a.n; ++j) {
            if (j > 0 && a.drafts) {
                const uint32_t id = (uint32_t)a.drafts[s * (a.n - 1) + j - 1];
                const uint32_t v = id < 0x80000000u ? id - (uint32_t)v0 : ~0u;
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    count[e] += v == (uint32_t)at(e);
                any |= v < (uint32_t)kLogitsPart;
            }
            const LogitsRaw<T, VEC> now = raw;
            if (j + 1 < a.n)
                raw.load(a, s * a.n + j + 1, v0, here);
            float x[8];
#pragma unroll
            for (int e = 0; e < 8; ++e)
                x[e] = (float)now.v[e];
            if (any != 0) {
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const float less = penalized(x[e], repetition);
                    x[e] = count[e] != 0 ? less : x[e];
                    const uint32_t said = count[e] & ~kLogitsPrompt;
                    const float told = (x[e] - frequency * (float)said) - presence;
                    x[e] = said != 0 ? told : x[e];
                }
            }
            if (biased != 0) {
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    if (biased >> e & 1u)
                        x[e] = x[e] + bias[e];
            }
#pragma unroll
            for (int e = 0; e < 8; ++e)
                if (!(now.allowed >> e & 1u))
                    x[e] = -__builtin_inff();
            T* const q = static_cast<T*>(a.out) + (s * a.n + j) * a.ld_out + v0;
            if (VEC && threadIdx.x * 8 + 8 <= here) {
                typename Vec8<T>::type r;
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    r[e] = (T)in_fp32<T>(x[e]);
                __builtin_nontemporal_store(r, reinterpret_cast<typename Vec8<T>::type*>(q + threadIdx.x * 8));
            } else {
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    if ((uint32_t)at(e) < here)
                        q[at(e)] = (T)in_fp32<T>(x[e]);
            }
        }
        __syncthreads();
    }
}

}  // namespace spk
