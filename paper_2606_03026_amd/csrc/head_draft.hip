// Host side of the verification of drafted tokens (C ABI in
// include/head_draft.h): validation, the split of the rows, two launches.
#include "head_draft.h"

#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstdint>

#include "draft.hpp"
#include "errors.hpp"

static_assert(2 * DRAFT_MAX_G + 1 <= spk::kDraftMaxRows, "every row of a sequence has a slot");

namespace {

using spk::aligned_to;
using spk::fail;
using spk::hip_fail;

constexpr int64_t kStatsWgs = 4096, kRaceWgs = 1024;

// Parts a row of V logits is cut into, where `rows` rows are worked on at once
// and `want` workgroups are to share them; whole stretches of 2,048 logits each.
void split(int64_t rows, int64_t want, int32_t V, int* parts, int* len)
{
    const int64_t stretches = ((int64_t)V + spk::kDraftStretch - 1) / spk::kDraftStretch;
    const int64_t most = std::min<int64_t>(
        {std::max<int64_t>(1, want / std::max<int64_t>(rows, 1)), stretches, (int64_t)spk::kDraftMaxParts});
    const int64_t per = (stretches + most - 1) / most;
    *parts = (int)((stretches + per - 1) / per);
    *len = (int)std::min<int64_t>(per * spk::kDraftStretch, (int64_t)1 << 30);
}

struct Plan {
    int rows, parts, part_len, race_parts, race_len;
    int64_t best_bytes, bytes;
};

bool sizes_ok(int32_t S, int32_t G, int32_t V)
{
    return S >= 0 && S <= DRAFT_MAX_S && G >= 0 && G <= DRAFT_MAX_G && V >= 1 && V <= DRAFT_MAX_V;
}

Plan make_plan(int32_t S, int32_t G, int32_t V, bool dist)
{
    Plan p{};
    p.rows = G + 1 + (dist ? G : 0);
    split((int64_t)S * p.rows, kStatsWgs, V, &p.parts, &p.part_len);
    split(S, kRaceWgs, V, &p.race_parts, &p.race_len);
    p.best_bytes = (int64_t)sizeof(spk::DraftBest) * S;
    p.bytes = p.best_bytes + (int64_t)sizeof(spk::DraftPart) * S * p.rows * p.parts;
    return p;
}

// (the race reads what the statistics wrote or cleared: it does not follow if they were refused)
template <typename T, int VEC>
hipError_t launch(const spk::DraftArgs& a, hipStream_t st)
{
    const dim3 block(spk::kDraftBlock), stats((unsigned)((int64_t)a.S * a.rows * a.parts)),
        race((unsigned)((int64_t)a.S * a.race_parts));
    if (a.part_len <= spk::kDraftStretch)
        hipLaunchKernelGGL((spk::k_draft_stats<T, VEC, 1>), stats, block, 0, st, a);
    else
        hipLaunchKernelGGL((spk::k_draft_stats<T, VEC, 2>), stats, block, 0, st, a);
    if (const hipError_t e = hipGetLastError(); e != hipSuccess)
        return e;
    if (a.race_len <= spk::kDraftStretch)
        hipLaunchKernelGGL((spk::k_draft_race<T, VEC, 1>), race, block, 0, st, a);
    else
        hipLaunchKernelGGL((spk::k_draft_race<T, VEC, 2>), race, block, 0, st, a);
    return hipGetLastError();
}

bool rows_vectorize(const void* p, int type, int64_t ld) { return aligned_to(p, 16) && ld * spk::type_bytes(type) % 16 == 0; }

}  // namespace

extern "C" {

int64_t head_draft_workspace_bytes(int32_t S, int32_t G, int32_t V)
{
    if (!sizes_ok(S, G, V))
        return -1;
    return std::max(make_plan(S, G, V, true).bytes, make_plan(S, G, V, false).bytes);
}

int head_draft_verify(const void* target, int64_t ld_target, const void* draft, int64_t ld_draft, int32_t logits_type,
                      const int32_t* drafts, const int32_t* n_draft, const float* uniform, const float* noise,
                      int64_t ld_noise, const float* temperature, int32_t S, int32_t G, int32_t V, int32_t* tokens,
                      int32_t* n_accepted, float* accept, float* prob, void* workspace, int64_t workspace_bytes,
                      void* stream)
{
    spk::last_error.clear();
    if (!sizes_ok(S, G, V))
        return fail(SPIKE_EINVAL, "S = %d, G = %d, V = %d outside [0, %d], [0, %d], [1, %d]", S, G, V, DRAFT_MAX_S,
                    DRAFT_MAX_G, DRAFT_MAX_V);
    if (!spk::is_float_type(logits_type))
        return fail(SPIKE_EINVAL, "logits type %d is not F32, BF16 or F16", logits_type);
    if (ld_target < V || (draft && ld_draft < V) || ld_noise < V)
        return fail(SPIKE_EINVAL, "row strides %lld, %lld and %lld must be at least V = %d", (long long)ld_target,
                    (long long)ld_draft, (long long)ld_noise, V);
    if (S == 0)
        return SPIKE_OK;
    if (!target || !noise || !tokens || !n_accepted || !workspace || (G > 0 && (!drafts || !uniform)))
        return fail(SPIKE_EINVAL, "null pointer argument");
    const int b = spk::type_bytes(logits_type);
    if (!aligned_to(target, b) || !aligned_to(draft, b) || !aligned_to(drafts, 4) || !aligned_to(n_draft, 4) ||
        !aligned_to(uniform, 4) || !aligned_to(noise, 4) || !aligned_to(temperature, 4) || !aligned_to(tokens, 4) ||
        !aligned_to(n_accepted, 4) || !aligned_to(accept, 4) || !aligned_to(prob, 4))
        return fail(SPIKE_EINVAL, "a pointer is not aligned to its element");
    if (!aligned_to(workspace, 16))
        return fail(SPIKE_EINVAL, "the workspace must be 16-byte aligned");
    const int64_t need = head_draft_workspace_bytes(S, G, V);
    if (workspace_bytes < need)
        return fail(SPIKE_EINVAL, "workspace of %lld bytes, needs %lld", (long long)workspace_bytes, (long long)need);
    const bool dist = draft != nullptr && G > 0;
    const Plan p = make_plan(S, G, V, dist);
    spk::DraftArgs a{};
    a.target = target, a.draft = dist ? draft : nullptr, a.ld_target = ld_target, a.ld_draft = ld_draft;
    a.drafts = drafts, a.n_draft = n_draft, a.uniform = uniform, a.noise = noise, a.ld_noise = ld_noise;
    a.temperature = temperature, a.S = S, a.G = G, a.V = V, a.rows = p.rows;
    a.parts = p.parts, a.part_len = p.part_len, a.race_parts = p.race_parts, a.race_len = p.race_len;
    a.tokens = tokens, a.n_accepted = n_accepted, a.accept = accept, a.prob = prob;
    a.best = static_cast<spk::DraftBest*>(workspace);
    a.part = reinterpret_cast<spk::DraftPart*>(static_cast<char*>(workspace) + p.best_bytes);
    const bool vec = rows_vectorize(target, logits_type, ld_target) &&
                     (!dist || rows_vectorize(draft, logits_type, ld_draft)) &&
                     rows_vectorize(noise, SPIKE_TYPE_F32, ld_noise);
    const hipStream_t st = static_cast<hipStream_t>(stream);
    hipError_t e = hipSuccess;
    switch (logits_type) {
    case SPIKE_TYPE_F32: e = vec ? launch<float, 8>(a, st) : launch<float, 1>(a, st); break;
    case SPIKE_TYPE_BF16: e = vec ? launch<spk::bf16, 8>(a, st) : launch<spk::bf16, 1>(a, st); break;
    default: e = vec ? launch<spk::f16, 8>(a, st) : launch<spk::f16, 1>(a, st); break;
    }
    return e == hipSuccess ? SPIKE_OK : hip_fail(e, "draft verification launch");
}

}  // extern "C"
