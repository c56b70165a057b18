// Embedding lookup and the gradient of its table (C ABI in
// include/spike_embed.h).
//
// Lookup: one wave per token, its lanes along the row; bound by memory (the
// distinct rows read once, T rows written).
//
// Gradient, by sorted tokens: the ids are sorted with their positions (equal
// ids in ascending position), the sorted list is cut into runs of a fixed
// length, and a wave adds up a run's rows for a block of columns, writing a
// row whenever the id changes.  A row whose tokens lie in one run is written
// at once; the others leave one partial sum per run, joined afterwards in
// ascending order.  No atomics: the order of every sum is fixed by the ids.
// The rows that no token names are most of a table's bytes: they are zeroed by
// workgroups beside those of all three steps, since sorting and adding are
// bound by latency and zeroing by the memory's writes.
#pragma once

#include "types.hpp"

namespace spk {

constexpr int kEmbedBlock = 256;
constexpr uint32_t kNoToken = 0xffffffffu;  // key of a token outside the table: sorts last

template <typename ID>
__device__ inline uint32_t token_key(const ID* ids, int64_t t, int V)
{
    const ID id = ids[t];
    return id >= 0 && id < (ID)V ? (uint32_t)id : kNoToken;
}

// VEC: 8 where every row starts on a 16-byte (I8: 8-byte) boundary and holds
// whole vectors, else 1.  (2500 rows of 1536, FP32, 31 MB: 6.1 us, 5.0 TB/s.)
template <typename TI, typename TO, int VEC, typename ID>
__global__ __launch_bounds__(kEmbedBlock) void k_embed(const TI* __restrict__ table, const float* __restrict__ row_scale,
                                                       int V, int D, int64_t ld_table, const ID* __restrict__ ids,
                                                       int T, float scale, TO* __restrict__ out, int64_t ld_out)
{
    const int t = blockIdx.x * (kEmbedBlock / 64) + threadIdx.x / 64;
    if (t >= T)
        return;
    const uint32_t id = __builtin_amdgcn_readfirstlane(token_key(ids, t, V));
    const bool live = id != kNoToken;
    const TI* row = table + (live ? id : 0) * ld_table;
    const float rs = sizeof(TI) == 1 && live ? row_scale[id] : 1.0f;
    TO* to = out + (int64_t)t * ld_out;
    const int lane = threadIdx.x % 64;
    for (int d = lane * VEC; d < D; d += 64 * VEC) {
        if constexpr (VEC == 8) {
            f32x8 v = {};
            if (live) {
                v = load8(row + d);
                if (sizeof(TI) == 1)
                    v *= rs;
                v *= scale;
            }
            store8(to + d, v);
        } else {
            float v = 0.0f;
            if (live) {
                v = (float)row[d];
                if (sizeof(TI) == 1)
                    v *= rs;
                v *= scale;
            }
            to[d] = (TO)in_fp32<TO>(v);
        }
    }
}

// --- sorting ---------------------------------------------------------------

constexpr int kSortChunk = 2048;   // tokens sorted among themselves by counting
constexpr int kSortParts = 8;      // lanes that share one token's count
constexpr int kSortTokens = kEmbedBlock / kSortParts;
constexpr int kSortPartKeys = kSortChunk / kSortParts;
constexpr int kSortPartStride = kSortPartKeys + 4;  // the parts' reads fall into different LDS banks

// Rows [first, first + count) of a table whose rows of `bytes` bytes lie `step`
// bytes apart, to be zeroed by workgroups of kFillRows rows each, and as many again
// kFillWgs groups on: a launch has to stay below 2^32 threads, a table of 2^28 rows has not.
struct FillArgs {
    char* table;
    int64_t step, bytes;
    int first, count;
    int wide;  // rows in 16-byte pieces, else in 2-byte ones
};

constexpr int kFillRows = 8;
constexpr int kFillWgs = 1 << 20;  // the most workgroups that zero rows in a launch
inline int fill_wgs(const FillArgs& f) { return f.count / kFillRows < kFillWgs ? (f.count + kFillRows - 1) / kFillRows : kFillWgs; }

__device__ inline void zero_row(const FillArgs& f, int row)
{
    char* p = f.table + row * f.step;
    if (f.wide)
        for (int64_t i = threadIdx.x % 64 * 16; i < f.bytes; i += 64 * 16)
            __builtin_nontemporal_store(u32x4{}, reinterpret_cast<u32x4*>(p + i));
    else
        for (int64_t i = threadIdx.x % 64 * 2; i < f.bytes; i += 64 * 2)
            *reinterpret_cast<uint16_t*>(p + i) = 0;
}

// All of this workgroup's rows.
__device__ inline void zero_rows(const FillArgs& f, int wg)
{
    for (int row0 = wg * kFillRows; row0 < f.count; row0 += kFillWgs * kFillRows)
        for (int r = row0 + threadIdx.x / 64; r < row0 + kFillRows && r < f.count; r += kEmbedBlock / 64)
            zero_row(f, f.first + r);
}

// Those of a group's rows that none of the T sorted keys names.
__device__ inline void zero_unnamed_group(const FillArgs& f, int wg, const uint32_t* __restrict__ keys, int T)
{
    __shared__ int named[kFillRows];
    const int v0 = f.first + wg * kFillRows;
    if (threadIdx.x < kFillRows)
        named[threadIdx.x] = 0;
    // the first of the sorted keys that is not below v0: 256 probes at a time
    int lo = 0, hi = T;  // keys before lo are below v0, keys from hi on are not
    while (hi > lo) {
        const int each = (hi - lo + kEmbedBlock - 1) / kEmbedBlock;
        const int at = lo + (int)threadIdx.x * each;
        const int below = __syncthreads_count(at < hi && keys[at] < (uint32_t)v0);
        // probes 0 .. below - 1 are below v0
        hi = below == 0 ? lo : min(hi, lo + below * each);
        lo = below == 0 ? lo : lo + (below - 1) * each + 1;
    }
    // mark the rows that come from there on
    for (int i = lo;; i += kEmbedBlock) {
        const int at = i + (int)threadIdx.x;
        const uint32_t row = at < T ? keys[at] - (uint32_t)v0 : kFillRows;
        if (row < kFillRows)
            named[row] = 1;
        if (__syncthreads_or(row >= kFillRows))
            break;
    }
    for (int r = threadIdx.x / 64; r < kFillRows && wg * kFillRows + r < f.count; r += kEmbedBlock / 64)
        if (!named[r])
            zero_row(f, v0 + r);
}

__device__ inline void zero_unnamed_rows(const FillArgs& f, int wg, const uint32_t* __restrict__ keys, int T)
{
    for (int group = wg; group * kFillRows < f.count; group += kFillWgs) {
        zero_unnamed_group(f, group, keys, T);
        __syncthreads();  // (its marks are read)
    }
}

// Sorts each chunk of kSortChunk tokens by (key, position): a token's place
// is the number of tokens of its chunk that come before it.  2,048
// comparisons a token, shared by 8 lanes.  Workgroups from sort_wgs on zero rows.
// (16,384 tokens and 108 MB of zeros: 20 us; bound by the memory's writes.)
template <typename ID>
__global__ __launch_bounds__(kEmbedBlock) void k_embed_sort(const ID* __restrict__ ids, int T, int V,
                                                            uint32_t* __restrict__ keys, int* __restrict__ order,
                                                            int sort_wgs, FillArgs fill)
{
    if ((int)blockIdx.x >= sort_wgs)
        return zero_rows(fill, blockIdx.x - sort_wgs);
    __shared__ uint32_t s[kSortParts * kSortPartStride];
    const int t0 = blockIdx.x * kSortTokens;
    const int c0 = t0 / kSortChunk * kSortChunk;
    const int n = min(kSortChunk, T - c0);
    uint32_t mine[kSortChunk / kEmbedBlock];
#pragma unroll
    for (int k = 0; k < kSortChunk / kEmbedBlock; ++k)
        mine[k] = token_key(ids, c0 + min(k * kEmbedBlock + (int)threadIdx.x, n - 1), V);
#pragma unroll
    for (int k = 0; k < kSortChunk / kEmbedBlock; ++k) {
        const int i = k * kEmbedBlock + threadIdx.x;
        s[i / kSortPartKeys * kSortPartStride + i % kSortPartKeys] = i < n ? mine[k] : kNoToken;
    }
    __syncthreads();
    const int part = threadIdx.x % kSortParts;
    const int i = t0 - c0 + threadIdx.x / kSortParts;  // this token's place in the chunk
    const uint32_t key = s[i / kSortPartKeys * kSortPartStride + i % kSortPartKeys];
    const uint32_t* p = s + part * kSortPartStride;
    const int j0 = part * kSortPartKeys;
    // of the equal keys, those at earlier places: `key + 1` bounds them up to place i, `key` from there on
    int before = 0;
    const int upto = i - j0;
#pragma unroll 8
    for (int j = 0; j < kSortPartKeys; j += 4) {
        const u32x4 k = *reinterpret_cast<const u32x4*>(p + j);
#pragma unroll
        for (int e = 0; e < 4; ++e)
            before += j + e < upto ? k[e] <= key : k[e] < key;
    }
    for (int m = 1; m < kSortParts; m *= 2)
        before += __shfl_xor(before, m);
    if (part == 0 && i < n) {
        keys[c0 + before] = key;
        order[c0 + before] = c0 + i;
    }
}

// Places every token of the sorted chunks in the whole list: its place in its
// own chunk, plus what the others hold before it (their equal keys too where
// they lie earlier), found by bisection.  8 lanes share a token's chunks.  Bound by the
// bisection's dependent reads, from the caches (16,384 tokens, with 44 MB of zeros: 9 us).
__global__ __launch_bounds__(kEmbedBlock) void k_embed_merge(const uint32_t* __restrict__ keys,
                                                             const int* __restrict__ order, int T,
                                                             uint32_t* __restrict__ out_keys,
                                                             int* __restrict__ out_order, int merge_wgs, FillArgs fill)
{
    if ((int)blockIdx.x >= merge_wgs)
        return zero_rows(fill, blockIdx.x - merge_wgs);
    const int i = blockIdx.x * kSortTokens + threadIdx.x / kSortParts;
    const int part = threadIdx.x % kSortParts;
    const bool live = i < T;
    const uint32_t key = live ? keys[i] : 0;
    const int own = i / kSortChunk;
    const int chunks = (T + kSortChunk - 1) / kSortChunk;
    int place = 0;
    if (live)
        for (int c = part; c < chunks; c += kSortParts) {
            if (c == own) {
                place += i - own * kSortChunk;
                continue;
            }
            // keys below, or up to, this one
            const uint32_t* p = keys + (int64_t)c * kSortChunk;
            int lo = 0, hi = min(kSortChunk, T - c * kSortChunk);
            while (lo < hi) {
                const int mid = (lo + hi) / 2;
                const uint32_t k = p[mid];
                if (k < key || (k == key && c < own))
                    lo = mid + 1;
                else
                    hi = mid;
            }
            place += lo;
        }
    for (int m = 1; m < kSortParts; m *= 2)
        place += __shfl_xor(place, m);
    if (live && part == 0) {
        out_keys[place] = key;
        out_order[place] = order[i];
    }
}

// --- sums ------------------------------------------------------------------

template <typename T, int VEC>
__device__ inline void load_cols(const T* p, float (&v)[VEC])
{
    typedef T tv __attribute__((ext_vector_type(VEC), aligned(VEC * sizeof(T) < 16 ? VEC * sizeof(T) : 16)));
    if constexpr (VEC > 1) {
        const tv x = *reinterpret_cast<const tv*>(p);
#pragma unroll
        for (int e = 0; e < VEC; ++e)
            v[e] = (float)x[e];
    } else {
        v[0] = (float)p[0];
    }
}

template <typename T, int VEC>
__device__ inline void put_row(T* p, const float (&v)[VEC], float scale, bool accumulate)
{
    typedef T tv __attribute__((ext_vector_type(VEC), aligned(VEC * sizeof(T) < 16 ? VEC * sizeof(T) : 16)));
    float x[VEC] = {};
    if (accumulate)
        load_cols<T, VEC>(p, x);
#pragma unroll
    for (int e = 0; e < VEC; ++e)
        x[e] = in_fp32<T>(v[e] * scale + x[e]);
    if constexpr (VEC > 1) {
        tv y;
#pragma unroll
        for (int e = 0; e < VEC; ++e)
            y[e] = (T)x[e];
        *reinterpret_cast<tv*>(p) = y;
    } else {
        p[0] = (T)x[0];
    }
}

// Tokens of a run; its keys and its two neighbours lie along the lanes of a wave.  A 352 MB
// table's gradient by 12, 16, 24 and 32 tokens: 2,500 tokens 68, 67, 68, 68 us; 16,384
// 87, 82, 81, 84; 60,000 tokens of a 32,000 x 256 table 88, 82, 78, 76.
constexpr int kRun = 24;
static_assert(kRun + 2 <= 64, "a run's keys lie along a wave");

// Workgroups below sum_wgs: each wave adds up one run (kRun tokens of the
// sorted list) for 64 VEC columns.  partial[2 r] holds run r's sum of a row that began in an
// earlier run, partial[2 r + 1] that of a row that begins in run r and goes
// on.  The other workgroups zero the rows that no token names.  Bound by memory: 16,384
// BF16 rows of 1536 read and 192 MB written, most of it zeros: 43 us, 5.6 TB/s.
template <typename TG, typename TD, int VEC>
__global__ __launch_bounds__(kEmbedBlock) void k_embed_sum(const TG* __restrict__ grad, int64_t ld_grad,
                                                           const uint32_t* __restrict__ keys,
                                                           const int* __restrict__ order, int T, int D,
                                                           int sum_wgs, float scale, int accumulate,
                                                           TD* __restrict__ dtable, int64_t ld_table,
                                                           float* __restrict__ partial, FillArgs fill)
{
    if ((int)blockIdx.x >= sum_wgs)
        return zero_unnamed_rows(fill, blockIdx.x - sum_wgs, keys, T);
    const int blocks = (D + 64 * VEC - 1) / (64 * VEC), lane = threadIdx.x % 64;
    const int unit = __builtin_amdgcn_readfirstlane(blockIdx.x * (kEmbedBlock / 64) + threadIdx.x / 64);
    const int r = unit / blocks;
    const int i0 = r * kRun;
    if (i0 >= T)
        return;
    const int n = min(kRun, T - i0);
    // column offset; lanes past the row repeat its last columns and store nothing
    const int col = (unit % blocks * 64 + lane) * VEC;
    const bool inside = col < D;
    const int d = inside ? col : D - VEC;
    // lane l holds the key before the run (l = 0) and those of its tokens (l = 1 .. n), then the one behind it
    const int at = i0 + lane - 1;
    const uint32_t key_l = lane <= n + 1 && at >= 0 && at < T ? keys[at] : kNoToken;
    const int order_l = lane >= 1 && lane <= n && key_l != kNoToken ? order[at] : 0;
    auto key_of = [&](int i) { return (uint32_t)__builtin_amdgcn_readlane(key_l, i + 1); };  // token i of the run; -1, n: its neighbours
    float sum[VEC] = {};
    bool from_before = i0 > 0 && key_of(-1) == key_of(0);
    constexpr int U = 8;  // rows in flight
    for (int i = 0; i < n; i += U) {
        float g[U][VEC];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            // (a padding token's gradient is not read: row 0 in its place; past the run, the last token's)
            const int t = __builtin_amdgcn_readlane(order_l, min(i + u, n - 1) + 1);
            load_cols<TG, VEC>(grad + (int64_t)t * ld_grad + d, g[u]);
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (i + u >= n)
                break;
            const uint32_t key = key_of(i + u);
            if (key == kNoToken)
                break;  // nor do any after it name a row
#pragma unroll
            for (int e = 0; e < VEC; ++e)
                sum[e] += g[u][e];
            const bool ends = i0 + i + u + 1 >= T || key_of(i + u + 1) != key;
            if (!ends && i + u + 1 < n)
                continue;
            if (inside) {
                if (ends && !from_before)
                    put_row<TD, VEC>(dtable + (int64_t)key * ld_table + d, sum, scale, accumulate);
                else
                    put_row<float, VEC>(partial + (int64_t)(2 * r + (from_before ? 0 : 1)) * D + d, sum, 1.0f, false);
            }
#pragma unroll
            for (int e = 0; e < VEC; ++e)
                sum[e] = 0.0f;
            from_before = false;
        }
    }
}

// Joins the partial sums of the rows that several runs share: the wave of the
// run in which such a row begins adds the following runs' sums to its own.
// Workgroups from join_wgs on zero rows that no token names.  Bound by the reads that
// depend on each other (16,384 tokens, with 32 MB written: 8.8 us).
template <typename TD, int VEC>
__global__ __launch_bounds__(kEmbedBlock) void k_embed_join(const uint32_t* __restrict__ keys, int T, int D,
                                                            float scale, int accumulate, TD* __restrict__ dtable,
                                                            int64_t ld_table, const float* __restrict__ partial,
                                                            int join_wgs, FillArgs fill)
{
    if ((int)blockIdx.x >= join_wgs)
        return zero_unnamed_rows(fill, blockIdx.x - join_wgs, keys, T);
    const int blocks = (D + 64 * VEC - 1) / (64 * VEC), lane = threadIdx.x % 64;
    const int unit = __builtin_amdgcn_readfirstlane(blockIdx.x * (kEmbedBlock / 64) + threadIdx.x / 64);
    const int r = unit / blocks;
    const int col = (unit % blocks * 64 + lane) * VEC;
    const bool inside = col < D;
    const int d = inside ? col : D - VEC;
    const int64_t i0 = (int64_t)r * kRun, i1 = i0 + kRun;
    if (i1 >= T)
        return;
    // lane 0: the key before this run; lane 1: its last; lane 2 + l: the first of the l-th run after it
    const int64_t at = lane == 0 ? i0 - 1 : lane == 1 ? i1 - 1 : i1 + (int64_t)(lane - 2) * kRun;
    uint32_t key_l = at >= 0 && at < T ? keys[at] : kNoToken;
    float sum[VEC];
    load_cols<float, VEC>(partial + (int64_t)(2 * r + 1) * D + d, sum);  // (asked for with the keys; there if a row goes on)
    const uint32_t key = __builtin_amdgcn_readlane(key_l, 1);
    if (key == kNoToken || (uint32_t)__builtin_amdgcn_readlane(key_l, 2) != key)
        return;  // no row goes on
    if (i0 > 0 && (uint32_t)__builtin_amdgcn_readlane(key_l, 0) == key)
        return;  // it began earlier
    constexpr int U = 8;  // partial sums in flight
    int64_t q = r + 1;    // the run whose key lane 2 holds
    for (;;) {
        // runs q .. q + more - 1 belong to the row
        const uint64_t differ = __ballot(lane >= 2 && key_l != key) >> 2;
        const int more = differ ? __builtin_ctzll(differ) : 62;
        for (int k = 0; k < more; k += U) {
            float p[U][VEC];
#pragma unroll
            for (int u = 0; u < U; ++u)
                load_cols<float, VEC>(partial + 2 * (q + min(k + u, more - 1)) * D + d, p[u]);
#pragma unroll
            for (int u = 0; u < U; ++u)
                if (k + u < more)
#pragma unroll
                    for (int e = 0; e < VEC; ++e)
                        sum[e] += p[u][e];
        }
        if (more < 62)
            break;
        q += 62;
        const int64_t next = q * kRun + (int64_t)(lane - 2) * kRun;
        key_l = lane >= 2 && next < T ? keys[next] : kNoToken;
    }
    if (inside)
        put_row<TD, VEC>(dtable + (int64_t)key * ld_table + d, sum, scale, accumulate);
}

}  // namespace spk
