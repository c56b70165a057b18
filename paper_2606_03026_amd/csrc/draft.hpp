// Verification of drafted tokens (C ABI in include/head_draft.h): a pass over
// every row of logits for its largest value and the sum of its exponentials,
// in parts of a row, then one workgroup per part of a sequence's decisive row
// decides on the drafts and races the residual.  The first is bound by memory
// where rows are many, by latency where they are few; the second by a chain of
// dependent loads, which it keeps short.
#pragma once

#include <math.h>

#include "types.hpp"

namespace spk {

constexpr int kDraftBlock = 256;
constexpr int kDraftStretch = kDraftBlock * 8;  // logits a workgroup takes at a time: 8 a thread
constexpr int kDraftMaxRows = 64;   // rows of one sequence: G + 1 of the target, G of the draft
constexpr int kDraftMaxParts = 64;  // parts of a row

// What a part of a row holds: its largest logit (-inf: none), that one's lowest
// index, and the sum of exp((x - top) / T) over the part.
struct DraftPart {
    float top;
    int at;
    float sum;
};

// Per sequence, for the race: the best r(v) / noise(v), or where r is zero throughout the
// best p(v) / noise(v), as a code that is larger the better the value and, of equal
// values, the lower v; upper half without its sign 0: none.  `done` counts the workgroups that have added theirs.
struct DraftBest {
    unsigned long long code;
    unsigned int done, pad;
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

__device__ inline float draft_nan_low(float x) { return fmaxf(x, -INFINITY); }  // (the maximum leaves a NaN out)

// Whether the temperature takes the largest logit alone, and log2(e) / T: at least
// the smallest normal number, so that an infinite difference stays infinite.
__device__ inline bool draft_greedy(float t) { return !(t > 0.0f); }
__device__ inline float draft_rate(float t) { return draft_greedy(t) ? 1.0f : fmaxf(1.44269504f / t, 1.17549435e-38f); }

// exp((x - top) / T): exactly 1 at the top (an infinite one too: the minimum leaves
// the difference's NaN out), 0 for -inf.
__device__ inline float draft_term(float x, float top, float rate)
{
    return __builtin_amdgcn_exp2f(fminf((x - top) * rate, 0.0f));
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

// Reductions over a full wave, every lane getting the result: within quads and rows
// of 16 by DPP moves, then the four rows' through scalar registers (a chain of
// shuffles through LDS takes several times as long).
template <int CTRL>
__device__ inline int draft_dpp(int v) { return __builtin_amdgcn_update_dpp(v, v, CTRL, 0xf, 0xf, false); }
constexpr int kQuadXor1 = 0xb1, kQuadXor2 = 0x4e, kRowRor4 = 0x124, kRowRor8 = 0x128;

template <int CTRL>
__device__ inline float draft_dpp(float v) { return __int_as_float(draft_dpp<CTRL>(__float_as_int(v))); }

__device__ inline float draft_row_of(float v, int row) { return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(v), 16 * row)); }

__device__ inline float draft_wave_max(float v)
{
    v = fmaxf(v, draft_dpp<kQuadXor1>(v));
    v = fmaxf(v, draft_dpp<kQuadXor2>(v));
    v = fmaxf(v, draft_dpp<kRowRor4>(v));
    v = fmaxf(v, draft_dpp<kRowRor8>(v));
    return fmaxf(fmaxf(draft_row_of(v, 0), draft_row_of(v, 1)), fmaxf(draft_row_of(v, 2), draft_row_of(v, 3)));
}

__device__ inline float draft_wave_sum(float v)
{
    v += draft_dpp<kQuadXor1>(v);
    v += draft_dpp<kQuadXor2>(v);
    v += draft_dpp<kRowRor4>(v);
    v += draft_dpp<kRowRor8>(v);
    return (draft_row_of(v, 0) + draft_row_of(v, 1)) + (draft_row_of(v, 2) + draft_row_of(v, 3));
}

__device__ inline int draft_wave_min(int v)
{
    v = min(v, draft_dpp<kQuadXor1>(v));
    v = min(v, draft_dpp<kQuadXor2>(v));
    v = min(v, draft_dpp<kRowRor4>(v));
    v = min(v, draft_dpp<kRowRor8>(v));
    return min(min(__builtin_amdgcn_readlane(v, 0), __builtin_amdgcn_readlane(v, 16)),
               min(__builtin_amdgcn_readlane(v, 32), __builtin_amdgcn_readlane(v, 48)));
}

template <int CTRL>
__device__ inline unsigned long long draft_dpp_max(unsigned long long v)
{
    const unsigned long long o = (unsigned long long)(uint32_t)draft_dpp<CTRL>((int)(v >> 32)) << 32 | (uint32_t)draft_dpp<CTRL>((int)v);
    return max(v, o);
}

__device__ inline unsigned long long draft_wave_max(unsigned long long v)
{
    v = draft_dpp_max<kQuadXor1>(v);
    v = draft_dpp_max<kQuadXor2>(v);
    v = draft_dpp_max<kRowRor4>(v);
    v = draft_dpp_max<kRowRor8>(v);
    unsigned long long r[4];
#pragma unroll
    for (int i = 0; i < 4; ++i)
        r[i] = (unsigned long long)(uint32_t)__builtin_amdgcn_readlane((int)(v >> 32), 16 * i) << 32 |
               (uint32_t)__builtin_amdgcn_readlane((int)v, 16 * i);
    return max(max(r[0], r[1]), max(r[2], r[3]));
}

// Joins one part per lane: every lane gets the whole.  Only a greedy row needs `at`,
// only the others their sum.
__device__ inline DraftPart draft_join(const DraftPart& mine, bool greedy, float rate)
{
    DraftPart all;
    all.top = draft_wave_max(mine.top);
    all.at = 0x7fffffff;
    all.sum = 0.0f;
    if (greedy) {
        all.at = draft_wave_min(mine.top == all.top ? mine.at : 0x7fffffff);
    } else {
        all.sum = draft_wave_sum(mine.top == -INFINITY ? 0.0f : mine.sum * draft_term(mine.top, all.top, rate));
    }
    return all;
}

// This thread's logits of ROUNDS stretches from `first` on, -inf from `end` on, as they
// are stored: a conversion or a choice between values here would wait for each stretch
// before the next is asked for (64 sequences of 57,344 logits: 30.5 us so, 29.3).
template <int VEC, int ROUNDS, typename T>
__device__ inline void draft_load(const T* row, int first, int end, typename Vec8<T>::type (&x)[ROUNDS])
{
#pragma unroll
    for (int r = 0; r < ROUNDS; ++r) {
        const int i = first + r * kDraftStretch + (int)threadIdx.x * 8;
        if (VEC == 8 && first + (r + 1) * kDraftStretch <= end) {
            x[r] = *reinterpret_cast<const typename Vec8<T>::type*>(row + i);
            continue;
        }
        x[r] = (T)-INFINITY;
        if (VEC == 8 && end % 8 == 0) {
            if (i < end)
                x[r] = *reinterpret_cast<const typename Vec8<T>::type*>(row + i);
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e)
                if (i + e < end)
                    x[r][e] = row[i + e];
        }
    }
}

// One workgroup per (part, row, sequence).  A thread takes 8 logits of each of
// ROUNDS stretches of 2,048 at a time, all loads in flight, then the largest of
// them, then their exponentials: one exponential per logit.  Bound by memory (64
// sequences of up to 4 drafts, 57,344 FP32 logits, 73 MB: 14.9 us, 4.9 TB/s), for one
// sequence by latency (3.4 us).
template <typename T, int VEC, int ROUNDS>
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
    const float rate = draft_rate(temp);
    const int i1 = min(a.V, (part + 1) * a.part_len);
    DraftPart me{-INFINITY, 0x7fffffff, 0.0f};
    for (int first = part * a.part_len; first < i1; first += ROUNDS * kDraftStretch) {
        typename Vec8<T>::type raw[ROUNDS];
        draft_load<VEC, ROUNDS>(x, first, i1, raw);
        const int i = first + (int)threadIdx.x * 8;
        float v[ROUNDS][8];
#pragma unroll
        for (int r = 0; r < ROUNDS; ++r)
#pragma unroll
            for (int e = 0; e < 8; ++e)
                v[r][e] = draft_nan_low((float)raw[r][e]);
        float top = me.top;
#pragma unroll
        for (int r = 0; r < ROUNDS; ++r)
#pragma unroll
            for (int e = 0; e < 8; ++e)
                top = fmaxf(top, v[r][e]);
        if (top == -INFINITY)
            continue;
        if (greedy) {
            if (top > me.top) {
                int at = 0x7fffffff;
#pragma unroll
                for (int r = ROUNDS - 1; r >= 0; --r)
#pragma unroll
                    for (int e = 7; e >= 0; --e)
                        at = v[r][e] == top ? i + r * kDraftStretch + e : at;
                me.top = top, me.at = at;
            }
            continue;
        }
        float sum = me.top == -INFINITY ? 0.0f : me.sum * draft_term(me.top, top, rate);
#pragma unroll
        for (int r = 0; r < ROUNDS; ++r)
#pragma unroll
            for (int e = 0; e < 8; ++e)
                sum += draft_term(v[r][e], top, rate);
        me.top = top, me.sum = sum;
    }
    __shared__ DraftPart s_part[kDraftBlock / 64];
    me = draft_join(me, greedy, rate);
    if (threadIdx.x % 64 == 0)
        s_part[threadIdx.x / 64] = me;
    __syncthreads();
    if (threadIdx.x < 64) {
        me = threadIdx.x < kDraftBlock / 64 ? s_part[threadIdx.x] : DraftPart{-INFINITY, 0x7fffffff, 0.0f};
        me = draft_join(me, greedy, rate);
        if (threadIdx.x == 0)
            a.part[((int64_t)s * a.rows + row) * a.parts + part] = me;
    }
}

// A row's distribution: p(v) = term * scale (scale = 1 / sum), or one at `at` (T = 0 and given drafts).
struct DraftDist {
    float top, scale;
    int at;
};

__device__ inline float draft_prob(const DraftDist& d, float x, int v, bool hot, float rate)
{
    if (hot)
        return v == d.at ? 1.0f : 0.0f;
    return x == -INFINITY ? 0.0f : draft_term(x, d.top, rate) * d.scale;
}

// A token of the residual goes before every other, one that its noise keeps from winning
// (a score of 0) too: then r is not zero throughout.  No score is negative, so their bits
// are ordered as they are.
__device__ inline unsigned long long draft_code(float score, int v, bool residual)
{
    return (unsigned long long)(__float_as_uint(score) | (residual ? 0x80000000u : 0u)) << 32 | (uint32_t)~v;
}
__device__ inline int draft_token(unsigned long long code) { return (code >> 32 & 0x7fffffffu) ? (int)~(uint32_t)code : -1; }

// One workgroup per (part, sequence): each decides on the drafts, then races its part,
// ROUNDS stretches of 2,048 at a time, all loads of a kind in flight.  Bound by its chain
// of dependent reads and atomics: 7.6 us for one sequence, 15.0 for 64 (44 MB).
template <typename T, int VEC, int ROUNDS>
__global__ __launch_bounds__(kDraftBlock) void k_draft_race(DraftArgs a)
{
    const int part = blockIdx.x % a.race_parts, s = blockIdx.x / a.race_parts;
    const int lane = threadIdx.x % 64, w = threadIdx.x / 64;
    __shared__ DraftDist s_dist[kDraftMaxRows];
    __shared__ float s_p[kDraftMaxRows], s_q[kDraftMaxRows];
    __shared__ int s_draft[kDraftMaxRows];
    __shared__ int s_taken;
    // Draft i is thread i's.  What does not depend on the decision is asked for at
    // once: the drafts, their random numbers, and the first stretch of the noise.
    const int mine = threadIdx.x;
    const int d_any = mine < a.G ? a.drafts[(int64_t)s * a.G + mine] : -1;
    const float u = mine < a.G ? a.uniform[(int64_t)s * a.G + mine] : 0.0f;
    const float* noise = a.noise + (int64_t)s * a.ld_noise;
    const int i0 = part * a.race_len, i1 = min(a.V, (part + 1) * a.race_len);
    Vec8<float>::type e[ROUNDS];
    draft_load<VEC, ROUNDS>(noise, i0, i1, e);  // past the end: -inf, which never wins
    const int n = draft_count(a, s);
    const float temp = a.temperature ? a.temperature[s] : 1.0f;
    const bool greedy = draft_greedy(temp);
    const float rate = draft_rate(temp);
    const int d = mine < n ? d_any : -1;
    float xt = -INFINITY, xd = -INFINITY;
    if (mine < n) {
        s_draft[mine] = d;
        if (d >= 0 && d < a.V) {
            xt = (float)draft_row<T>(a, s, mine)[d];
            if (a.draft)
                xd = (float)draft_row<T>(a, s, a.G + 1 + mine)[d];
        }
    }
    // the rows' distributions: one wave per row, its parts along the lanes, four rows' loads at a time
    for (int r0 = w; r0 < a.rows; r0 += 4 * (kDraftBlock / 64)) {
        DraftPart me[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const int row = r0 + k * (kDraftBlock / 64);
            me[k] = DraftPart{-INFINITY, 0x7fffffff, 0.0f};
            if (row < a.rows && (row <= a.G ? row <= n : row - a.G - 1 < n) && lane < a.parts)
                me[k] = a.part[((int64_t)s * a.rows + row) * a.parts + lane];
        }
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const int row = r0 + k * (kDraftBlock / 64);
            if (row >= a.rows)
                break;
            const DraftPart all = draft_join(me[k], greedy, rate);
            if (lane == 0)
                s_dist[row] = DraftDist{all.top, 1.0f / all.sum, all.top == -INFINITY ? -1 : all.at};
        }
    }
    __syncthreads();
    if (w == 0) {
        float p = 0.0f, q = 0.0f;
        if (mine < n && d >= 0 && d < a.V) {
            p = draft_prob(s_dist[mine], draft_nan_low(xt), d, greedy, rate);
            q = a.draft ? draft_prob(s_dist[a.G + 1 + mine], draft_nan_low(xd), d, greedy, rate) : 1.0f;
        }
        if (mine < n) {
            s_p[mine] = p;
            s_q[mine] = q;
        }
        const unsigned long long refused = __ballot(mine < n && !(u * q < p));
        if (lane == 0)
            s_taken = refused ? __builtin_ctzll(refused) : n;
    }
    __syncthreads();
    const int j = s_taken;
    const T* target = draft_row<T>(a, s, j);
    const bool minus = j < n;  // a draft was refused: its distribution is taken off
    const T* draft = minus && a.draft ? draft_row<T>(a, s, a.G + 1 + j) : nullptr;
    const DraftDist dp = s_dist[j];
    const DraftDist dq = !minus ? DraftDist{0.0f, 1.0f, -1} : draft ? s_dist[a.G + 1 + j] : DraftDist{0.0f, 1.0f, s_draft[j]};
    const bool hot_q = greedy || !draft;
    unsigned long long best = 0;
    for (int first = i0; first < i1; first += ROUNDS * kDraftStretch) {
        typename Vec8<T>::type x[ROUNDS], y[ROUNDS];
        draft_load<VEC, ROUNDS>(target, first, i1, x);
        if (draft) {
            draft_load<VEC, ROUNDS>(draft, first, i1, y);
        } else {
#pragma unroll
            for (int r = 0; r < ROUNDS; ++r)
                y[r] = (T)-INFINITY;
        }
#pragma unroll
        for (int r = 0; r < ROUNDS; ++r)
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                const int v = first + r * kDraftStretch + (int)threadIdx.x * 8 + k;
                const float p = draft_prob(dp, draft_nan_low((float)x[r][k]), v, greedy, rate);
                const float left = p - draft_prob(dq, draft_nan_low((float)y[r][k]), v, hot_q, rate);
                const float inverse = e[r][k] > 0.0f ? __builtin_amdgcn_rcpf(e[r][k]) : 0.0f;
                const float score = fmaxf((left > 0.0f ? left : p) * inverse, 0.0f);  // (0 times infinity: 0)
                best = max(best, draft_code(score, v, left > 0.0f));
            }
        if (first + ROUNDS * kDraftStretch < i1)
            draft_load<VEC, ROUNDS>(noise, first + ROUNDS * kDraftStretch, i1, e);
    }
    best = draft_wave_max(best);
    __shared__ unsigned long long s_best[kDraftBlock / 64];
    __shared__ int s_last;
    if (lane == 0)
        s_best[w] = best;
    __syncthreads();
    if (threadIdx.x == 0) {
#pragma unroll
        for (int k = 1; k < kDraftBlock / 64; ++k)
            best = max(best, s_best[k]);
        DraftBest* b = a.best + s;
        int last = 1;
        if (a.race_parts > 1) {
            atomicMax(&b->code, best);
            // the maximum is at the device's point of coherence before the count is
            asm volatile("" ::: "memory");
            __builtin_amdgcn_s_waitcnt(0);
            asm volatile("" ::: "memory");
            last = atomicAdd(&b->done, 1u) == (unsigned)a.race_parts - 1;
            if (last)
                best = atomicMax(&b->code, 0ull);
        }
        s_last = last;
        s_best[0] = best;
    }
    __syncthreads();
    if (!s_last || mine > a.G)
        return;
    best = s_best[0];
    const int token = draft_token(best);
    const int64_t o = (int64_t)s * (a.G + 1) + mine;
    if (mine == 0)
        a.n_accepted[s] = j;
    a.tokens[o] = mine < j ? d : mine == j ? token : -1;
    if (a.prob)
        a.prob[o] = mine < j ? s_p[mine]
                    : mine == j && token >= 0 ? draft_prob(dp, draft_nan_low((float)target[token]), token, greedy, rate)
                                              : 0.0f;
    if (a.accept && mine < a.G) {
        const float p = mine < n ? s_p[mine] : 0.0f, q = mine < n ? s_q[mine] : 0.0f;
        a.accept[(int64_t)s * a.G + mine] = q > 0.0f ? fminf(p / q, 1.0f) : p > 0.0f ? 1.0f : 0.0f;
    }
}

}  // namespace spk
