// Verification of drafted tokens (C ABI in include/head_draft.h): a pass over
// every row of logits for its largest value and the sum of its exponentials,
// in parts of a row, then one workgroup per part of a sequence's decisive row
// decides on the drafts and races the residual.
#pragma once

#include <math.h>

#include "types.hpp"

namespace spk {

constexpr int kDraftBlock = 256;
constexpr int kDraftMaxRows = 64;   // rows of one sequence: G + 1 of the target, G of the draft
constexpr int kDraftMaxParts = 64;  // parts of a row

// What a part of a row holds: its largest logit (-inf: none), that one's lowest
// index, and the sum of exp((x - top) / T) over the part.
struct DraftPart {
    float top;
    int at;
    float sum;
};

// Per sequence, for the race: the best r(v) / noise(v) and p(v) / noise(v) as
// (value bits << 32 | ~v), so that the largest code is the largest value at
// the lowest index; 0: none.  `done` counts the workgroups that have added theirs.
struct DraftBest {
    unsigned long long r, p;
    unsigned int done, pad[3];
};

struct DraftArgs {
    const void *target, *draft;
    int64_t ld_target, ld_draft;
    const int32_t *drafts, *n_draft;
    const float *uniform, *noise;
    int64_t ld_noise;
    const float* temperature;
    int S, G, V;
    int rows;   // per sequence: G + 1, and G more with a draft distribution
    int parts, part_len;            // the statistics: parts of a row, logits of a part
    int race_parts, race_len;       // the race
    int32_t *tokens, *n_accepted;
    float *accept, *prob;
    DraftPart* part;  // [S][rows][parts]
    DraftBest* best;  // [S]
};

__device__ inline float draft_nan_low(float x) { return x == x ? x : -INFINITY; }

// Whether the temperature takes the largest logit alone, and 1 / T: at least
// the smallest normal number, so that an infinite difference stays infinite.
__device__ inline bool draft_greedy(float t) { return !(t > 0.0f); }
__device__ inline float draft_inverse(float t) { return draft_greedy(t) ? 1.0f : fmaxf(1.0f / t, 1.17549435e-38f); }

// exp((x - top) / T): exactly 1 at the top (an infinite one too), 0 for -inf.
__device__ inline float draft_term(float x, float top, float inv_t)
{
    return x == top ? 1.0f : expf((x - top) * inv_t);
}

__device__ inline int draft_count(const DraftArgs& a, int s)
{
    return a.n_draft ? min(max(a.n_draft[s], 0), a.G) : a.G;
}

// Row `row` of sequence s: the target's G + 1, then the draft's G.
template <typename T>
__device__ inline const T* draft_row(const DraftArgs& a, int s, int row)
{
    return row <= a.G ? static_cast<const T*>(a.target) + ((int64_t)s * (a.G + 1) + row) * a.ld_target
                      : static_cast<const T*>(a.draft) + ((int64_t)s * a.G + row - a.G - 1) * a.ld_draft;
}

__device__ inline void draft_join(DraftPart& a, const DraftPart& b, float inv_t)
{
    const bool b_wins = b.top > a.top || (b.top == a.top && b.at < a.at);
    const float top = b_wins ? b.top : a.top;
    const float sum = top == -INFINITY ? 0.0f
                                       : a.sum * (a.top == -INFINITY ? 0.0f : draft_term(a.top, top, inv_t)) +
                                             b.sum * (b.top == -INFINITY ? 0.0f : draft_term(b.top, top, inv_t));
    a = DraftPart{top, b_wins ? b.at : a.at, sum};
}

template <typename T, int VEC>
__device__ inline void draft_load(const T* row, int i, int end, float (&x)[8])
{
    if (VEC == 8 && i + 8 <= end) {
        const f32x8 v = load8(row + i);
        for (int e = 0; e < 8; ++e)
            x[e] = draft_nan_low(v[e]);
    } else {
        for (int e = 0; e < 8; ++e)
            x[e] = i + e < end ? draft_nan_low((float)row[i + e]) : -INFINITY;
    }
}

// One workgroup per (part, row, sequence).
template <typename T, int VEC>
__global__ __launch_bounds__(kDraftBlock) void k_draft_stats(DraftArgs a)
{
    const int part = blockIdx.x % a.parts, row = blockIdx.x / a.parts % a.rows, s = blockIdx.x / a.parts / a.rows;
    if (part == 0 && row == 0 && threadIdx.x == 0)
        a.best[s] = DraftBest{};
    const int n = draft_count(a, s);
    if (row <= a.G ? row > n : row - a.G - 1 >= n)
        return;  // past the sequence's drafts
    const T* x = draft_row<T>(a, s, row);
    const float temp = a.temperature ? a.temperature[s] : 1.0f;
    const bool greedy = draft_greedy(temp);
    const float inv_t = draft_inverse(temp);
    const int i0 = part * a.part_len, i1 = min(a.V, i0 + a.part_len);
    DraftPart me{-INFINITY, a.V, 0.0f};
    for (int i = i0 + (int)threadIdx.x * 8; i < i1; i += kDraftBlock * 8) {
        float v[8];
        draft_load<T, VEC>(x, i, i1, v);
        float top = v[0];
        int at = 0;
        for (int e = 1; e < 8; ++e)
            if (v[e] > top)
                top = v[e], at = e;
        if (top == -INFINITY)
            continue;
        float sum = 0.0f;
        if (!greedy)
            for (int e = 0; e < 8; ++e)
                sum += draft_term(v[e], top, inv_t);
        draft_join(me, DraftPart{top, i + at, sum}, inv_t);
    }
    __shared__ DraftPart s_part[kDraftBlock / 64];
    for (int m = 1; m < 64; m *= 2)
        draft_join(me, DraftPart{__shfl_xor(me.top, m), __shfl_xor(me.at, m), __shfl_xor(me.sum, m)}, inv_t);
    if (threadIdx.x % 64 == 0)
        s_part[threadIdx.x / 64] = me;
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int w = 1; w < kDraftBlock / 64; ++w)
            draft_join(me, s_part[w], inv_t);
        a.part[((int64_t)s * a.rows + row) * a.parts + part] = me;
    }
}

// A row's distribution: p(v) = term / sum, or one at `at` (T = 0 and given drafts).
struct DraftDist {
    float top, sum;
    int at;
};

__device__ inline float draft_prob(const DraftDist& d, float x, int v, bool hot, float inv_t)
{
    if (hot)
        return v == d.at ? 1.0f : 0.0f;
    return x == -INFINITY || d.top == -INFINITY ? 0.0f : draft_term(x, d.top, inv_t) / d.sum;
}

__device__ inline unsigned long long draft_code(float score, int v)
{
    return score > 0.0f ? (unsigned long long)__float_as_uint(score) << 32 | (uint32_t)~v : 0ull;
}

// One workgroup per (part, sequence): each decides on the drafts, then races its part.
template <typename T, int VEC>
__global__ __launch_bounds__(kDraftBlock) void k_draft_race(DraftArgs a)
{
    const int part = blockIdx.x % a.race_parts, s = blockIdx.x / a.race_parts;
    const int n = draft_count(a, s);
    const float temp = a.temperature ? a.temperature[s] : 1.0f;
    const bool greedy = draft_greedy(temp);
    const float inv_t = draft_inverse(temp);
    __shared__ DraftDist s_dist[kDraftMaxRows];
    __shared__ float s_p[kDraftMaxRows], s_q[kDraftMaxRows];
    __shared__ int s_taken;
    // the rows' distributions, one wave per row, its parts along the lanes
    for (int row = threadIdx.x / 64; row < a.rows; row += kDraftBlock / 64) {
        if (row <= a.G ? row > n : row - a.G - 1 >= n)
            continue;
        const int lane = threadIdx.x % 64;
        DraftPart me{-INFINITY, a.V, 0.0f};
        if (lane < a.parts)
            me = a.part[((int64_t)s * a.rows + row) * a.parts + lane];
        for (int m = 1; m < 64; m *= 2)
            draft_join(me, DraftPart{__shfl_xor(me.top, m), __shfl_xor(me.at, m), __shfl_xor(me.sum, m)}, inv_t);
        if (lane == 0)
            s_dist[row] = DraftDist{me.top, me.sum, me.top == -INFINITY ? -1 : me.at};
    }
    __syncthreads();
    if ((int)threadIdx.x < n) {
        const int i = threadIdx.x;
        const int d = a.drafts[(int64_t)s * a.G + i];
        float p = 0.0f, q = 0.0f;
        if (d >= 0 && d < a.V) {
            p = draft_prob(s_dist[i], draft_nan_low((float)draft_row<T>(a, s, i)[d]), d, greedy, inv_t);
            q = a.draft ? draft_prob(s_dist[a.G + 1 + i], draft_nan_low((float)draft_row<T>(a, s, a.G + 1 + i)[d]), d,
                                     greedy, inv_t)
                        : 1.0f;
        }
        s_p[i] = p;
        s_q[i] = q;
    }
    __syncthreads();
    if (threadIdx.x == 0) {
        int j = 0;
        while (j < n && a.uniform[(int64_t)s * a.G + j] * s_q[j] < s_p[j])
            ++j;
        s_taken = j;
    }
    __syncthreads();
    const int j = s_taken;
    const T* target = draft_row<T>(a, s, j);
    const bool minus = j < n;  // a draft was refused: its distribution is taken off
    const T* draft = minus && a.draft ? draft_row<T>(a, s, a.G + 1 + j) : nullptr;
    const DraftDist dp = s_dist[j];
    const DraftDist dq = !minus ? DraftDist{} : draft ? s_dist[a.G + 1 + j] : DraftDist{0.0f, 0.0f, a.drafts[(int64_t)s * a.G + j]};
    const bool hot_q = greedy || !draft;
    const float* noise = a.noise + (int64_t)s * a.ld_noise;
    unsigned long long best_r = 0, best_p = 0;
    const int i0 = part * a.race_len, i1 = min(a.V, i0 + a.race_len);
    for (int i = i0 + (int)threadIdx.x * 8; i < i1; i += kDraftBlock * 8) {
        float x[8], y[8], e[8];
        draft_load<T, VEC>(target, i, i1, x);
        if (draft)
            draft_load<T, VEC>(draft, i, i1, y);
        draft_load<float, VEC>(noise, i, i1, e);  // past the end: -inf, which never wins
        for (int k = 0; k < 8; ++k) {
            if (!(e[k] > 0.0f))
                continue;
            const int v = i + k;
            const float p = draft_prob(dp, x[k], v, greedy, inv_t);
            const float q = minus ? draft_prob(dq, draft ? y[k] : 0.0f, v, hot_q, inv_t) : 0.0f;
            best_p = max(best_p, draft_code(p / e[k], v));
            best_r = max(best_r, draft_code((p - q) / e[k], v));
        }
    }
    for (int m = 1; m < 64; m *= 2) {
        best_r = max(best_r, (unsigned long long)__shfl_xor(best_r, m));
        best_p = max(best_p, (unsigned long long)__shfl_xor(best_p, m));
    }
    __shared__ unsigned long long s_best[2][kDraftBlock / 64];
    if (threadIdx.x % 64 == 0) {
        s_best[0][threadIdx.x / 64] = best_r;
        s_best[1][threadIdx.x / 64] = best_p;
    }
    __syncthreads();
    if (threadIdx.x != 0)
        return;
    for (int w = 1; w < kDraftBlock / 64; ++w) {
        best_r = max(best_r, s_best[0][w]);
        best_p = max(best_p, s_best[1][w]);
    }
    DraftBest* b = a.best + s;
    atomicMax(&b->r, best_r);
    atomicMax(&b->p, best_p);
    // the maxima are at the device's point of coherence before the count is
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt(0);
    asm volatile("" ::: "memory");
    if (atomicAdd(&b->done, 1u) != (unsigned)a.race_parts - 1)
        return;
    best_r = atomicMax(&b->r, 0ull);
    best_p = atomicMax(&b->p, 0ull);
    const unsigned long long win = best_r ? best_r : best_p;
    const int token = win ? (int)~(uint32_t)win : -1;
    a.n_accepted[s] = j;
    for (int i = 0; i <= a.G; ++i) {
        const int64_t o = (int64_t)s * (a.G + 1) + i;
        a.tokens[o] = i < j ? a.drafts[(int64_t)s * a.G + i] : i == j ? token : -1;
        if (a.prob)
            a.prob[o] = i < j ? s_p[i]
                        : i == j && token >= 0 ? draft_prob(dp, draft_nan_low((float)target[token]), token, greedy, inv_t)
                                               : 0.0f;
        if (a.accept && i < a.G)
            a.accept[(int64_t)s * a.G + i] = i >= n ? 0.0f : s_q[i] > 0.0f ? fminf(s_p[i] / s_q[i], 1.0f) : s_p[i] > 0.0f ? 1.0f : 0.0f;
    }
}

}  // namespace spk
