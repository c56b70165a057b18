// Host side of the penalties, biases and masks on logits (C ABI in
// include/head_logits.h): validation and one launch.
#include "head_logits.h"

#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstdint>

#include "errors.hpp"
#include "logits.hpp"

namespace {

using spk::aligned_to;
using spk::fail;
using spk::hip_fail;

template <typename T>
void launch(const spk::LogitsArgs& a, bool vec, hipStream_t st)
{
    const dim3 grid((unsigned)std::min<int64_t>((int64_t)a.S * a.parts, 1 << 20));
    if (vec)
        hipLaunchKernelGGL((spk::k_logits<T, true>), grid, dim3(256), 0, st, a);
    else
        hipLaunchKernelGGL((spk::k_logits<T, false>), grid, dim3(256), 0, st, a);
}

}  // namespace

extern "C" {

int head_logits_adjust(const void* logits, int64_t ld_logits, int32_t type, int32_t S, int32_t n, int32_t V,
                       const int32_t* ids, int64_t ld_ids, int32_t L, const int32_t* n_ids, const int32_t* n_prompt,
                       const int32_t* drafts, const float* repetition, const float* presence, const float* frequency,
                       const int32_t* bias_ids, const float* bias, int32_t n_bias, const uint32_t* mask,
                       int64_t ld_mask, void* out, int64_t ld_out, void* stream)
{
    spk::last_error.clear();
    if (S < 0 || S > LOGITS_MAX_S || n < 1 || n > LOGITS_MAX_N || V < 1 || V > LOGITS_MAX_V)
        return fail(SPIKE_EINVAL, "S = %d, n = %d, V = %d outside [0, %d], [1, %d], [1, %d]", S, n, V, LOGITS_MAX_S,
                    LOGITS_MAX_N, LOGITS_MAX_V);
    if (L < 0 || L > LOGITS_MAX_L || n_bias < 0 || n_bias > LOGITS_MAX_BIAS)
        return fail(SPIKE_EINVAL, "L = %d, n_bias = %d outside [0, %d], [0, %d]", L, n_bias, LOGITS_MAX_L, LOGITS_MAX_BIAS);
    if (!spk::is_float_type(type))
        return fail(SPIKE_EINVAL, "logits type %d is not F32, BF16 or F16", type);
    if (ld_logits < V || ld_out < V || (ids && ld_ids < L) || (mask && ld_mask < ((int64_t)V + 31) / 32))
        return fail(SPIKE_EINVAL, "a row stride is below V = %d, L = %d or the words of a mask", V, L);
    if ((n_bias > 0 && (!bias_ids || !bias)))
        return fail(SPIKE_EINVAL, "%d biases without their tokens or values", n_bias);
    if (S == 0)
        return SPIKE_OK;
    if (!logits || !out)
        return fail(SPIKE_EINVAL, "null pointer (logits %p, out %p)", logits, out);
    if (out == logits && ld_out != ld_logits)
        return fail(SPIKE_EINVAL, "out is logits with another row stride");
    const int b = spk::type_bytes(type);
    if (!aligned_to(logits, b) || !aligned_to(out, b) || !aligned_to(ids, 4) || !aligned_to(n_ids, 4) ||
        !aligned_to(n_prompt, 4) || !aligned_to(drafts, 4) || !aligned_to(repetition, 4) || !aligned_to(presence, 4) ||
        !aligned_to(frequency, 4) || !aligned_to(bias_ids, 4) || !aligned_to(bias, 4) || !aligned_to(mask, 4))
        return fail(SPIKE_EINVAL, "a pointer is not aligned to its element");
    spk::LogitsArgs a{};
    a.logits = logits, a.ld_logits = ld_logits, a.S = S, a.n = n, a.V = V;
    a.ids = L > 0 ? ids : nullptr, a.ld_ids = ld_ids, a.L = L, a.n_ids = n_ids, a.n_prompt = n_prompt;
    a.drafts = drafts, a.repetition = repetition, a.presence = presence, a.frequency = frequency;
    a.bias_ids = bias_ids, a.bias = bias, a.n_bias = n_bias, a.mask = mask, a.ld_mask = ld_mask;
    a.out = out, a.ld_out = ld_out;
    a.parts = (int)(((int64_t)V + spk::kLogitsPart - 1) / spk::kLogitsPart);
    a.vec_ids = aligned_to(ids, 16) && ld_ids % 4 == 0;
    const bool vec = aligned_to(logits, 16) && aligned_to(out, 16) && ld_logits * b % 16 == 0 && ld_out * b % 16 == 0;
    const hipStream_t st = static_cast<hipStream_t>(stream);
    switch (type) {
    case SPIKE_TYPE_F32: launch<float>(a, vec, st); break;
    case SPIKE_TYPE_BF16: launch<spk::bf16>(a, vec, st); break;
    default: launch<spk::f16>(a, vec, st); break;
    }
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? SPIKE_OK : hip_fail(e, "logits launch");
}

}  // extern "C"
