// Four-bit weights of the fused projection (C ABI in include/dense_fused.h): their layout, and the
// products with rows of four-bit codes, on the matrix instructions that scale their operands' blocks.
#pragma once

#include "fused.hpp"

namespace spk {

// --- layout ----------------------------------------------------------------

// Exponents are kept relative to the largest of their output's blocks that are not all zero: that one becomes
// kMxTop, which F16 holds times 6, and the difference goes into the output's scale.  F16 operands then hold a weight to
// 2^-37 of its output's largest at worst and exactly where its block is within 2^-36 of the largest one.
constexpr int kMxTop = 127 + 13;

__device__ inline bool mx_row_in(const uint8_t* row, int64_t block, int K, uint32_t (&w)[4])
{
    // 16 bytes of codes of a block, those past K zero; any alignment
    uint32_t any = 0;
    for (int i = 0; i < 4; ++i) {
        w[i] = 0;
        for (int e = 0; e < 4; ++e) {
            const int64_t k = block * kMxBlock + 8 * i + 2 * e;
            if (k < K)
                w[i] |= (uint32_t)(row[k / 2] & (k + 1 < K ? 0xff : 0x0f)) << (8 * e);
        }
        any |= w[i] & 0x77777777u;  // (a zero has a sign)
    }
    return any != 0;
}

// An output's largest exponent, and its scale: a wave an output; top [n_out rounded up to 16], zeros past M.
__global__ __launch_bounds__(256) void k_mx4_top(const uint8_t* codes, int64_t ld_codes, const uint8_t* scales, int64_t ld_scales,
                                                 int K, int M, int padded, uint8_t* top, float* scale)
{
    const int m = blockIdx.x * 4 + threadIdx.x / 64;
    if (m >= padded)
        return;
    const int blocks = (K + kMxBlock - 1) / kMxBlock;
    int most = 0;
    for (int b = threadIdx.x % 64; m < M && b < blocks; b += 64) {
        uint32_t w[4];
        const int byte = scales[m * ld_scales + b];
        if (byte != 255 && byte > most && mx_row_in(codes + m * ld_codes, b, K, w))
            most = byte;
    }
#pragma unroll
    for (int d = 32; d > 0; d /= 2)
        most = max(most, __shfl_xor(most, d));
    if (threadIdx.x % 64 == 0) {
        const int e = most - kMxTop;  // 2^e, down to 2^-140
        top[m] = (uint8_t)most;
        scale[m] = m >= M ? 0.0f : __uint_as_float(e >= -126 ? (uint32_t)(e + 127) << 23 : 1u << (149 + e));
    }
}

// A block's exponent relative to its output's largest; -1: it and its codes count as zero (smaller than the largest by 2^-140).
__device__ inline int mx_relative(int byte, int top, bool any) { return byte == 255 ? 255 : any ? max(byte - top + kMxTop, -1) : -1; }

// [tiles][blocks, rounded up to 4][16 outputs][16 B] and [tiles][blocks / 4][16 outputs][4 B]; and the exponents once more in
// k_mx4_tile's order, [tiles][fours of 128 inputs][block of 128][16 outputs][4 B, one for each of the four].  A thread a block.
__global__ __launch_bounds__(256) void k_mx4_pack(const uint8_t* codes, int64_t ld_codes, const uint8_t* scales, int64_t ld_scales,
                                                  int K, int M, const uint8_t* top, uint8_t* P, uint8_t* S, uint8_t* E, int64_t total)
{
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (i >= total)
        return;
    const int64_t blocks = ((int64_t)K + 4 * kMxBlock - 1) / (4 * kMxBlock) * 4;
    const int c = i % 16;
    const int64_t block = i / 16 % blocks, tile = i / 16 / blocks, m = mx4_output(tile, c);
    uint32_t w[4] = {};
    int byte = -1;
    if (m < M && block * kMxBlock < K) {
        const bool any = mx_row_in(codes + m * ld_codes, block, K, w);
        byte = mx_relative(scales[m * ld_scales + block], top[m], any);
    }
    if (byte < 0)
        w[0] = w[1] = w[2] = w[3] = 0, byte = 127;
    *reinterpret_cast<u32x4*>(P + i * 16) = u32x4{w[0], w[1], w[2], w[3]};
    S[(tile * (blocks / 4) + block / 4) * 64 + c * 4 + block % 4] = (uint8_t)byte;
    E[(tile * ((blocks + 15) / 16) + block / 16) * 256 + (block % 4 * 16 + c) * 4 + block / 4 % 4] = (uint8_t)byte;
}

// The gradient's: columns as outputs, a weight times its output's kMxTop-relative scale as one E5M2 byte (exact
// where its block is within 2^-28 of the output's largest, else to 2^-29 of that), in k_fused_pack's order but for
// the outputs'.
__global__ __launch_bounds__(256) void k_mx4_pack_columns(const uint8_t* codes, int64_t ld_codes, const uint8_t* scales,
                                                          int64_t ld_scales, int K, int M, const uint8_t* top, int8_t* P, int64_t chunks)
{
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (i >= chunks)
        return;
    const int steps = (M + kFusedStep - 1) / kFusedStep;
    const int lane = i % 64;
    const int64_t piece = i / 64;
    const int64_t k = mx4_output(piece / steps, lane % 16), m0 = piece % steps * kFusedStep + lane / 16 * 8;
    uint32_t w[4];
    for (int r = 0; r < 4; ++r) {
        float v[4];
        for (int e = 0; e < 4; ++e) {
            const int j = 4 * r + e;
            const int64_t m = m0 + j % 8 + j / 8 * 32;
            v[e] = 0.0f;
            if (k < K && m < M) {
                const uint32_t code = codes[m * ld_codes + k / 2] >> (k % 2 * 4) & 15u;
                const int byte = mx_relative(scales[m * ld_scales + k / kMxBlock], top[m], (code & 7u) != 0);
                v[e] = byte < 0 ? 0.0f : __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(code, mx_scale((uint32_t)byte), 0)[0];
            }
        }
        w[r] = (uint32_t)__builtin_amdgcn_cvt_pk_bf8_f32(v[2], v[3], __builtin_amdgcn_cvt_pk_bf8_f32(v[0], v[1], 0, false), true);
    }
    reinterpret_cast<u32x4*>(P)[i] = u32x4{w[0], w[1], w[2], w[3]};
}

// --- products --------------------------------------------------------------

struct Mx4Args {
    FusedArgs f;  // (steps: of 128 inputs; x: the rows' codes, ld_x: bytes)
    const uint8_t* scales;
    int64_t ld_scales;
    const int8_t* E;  // the weights' exponents in k_mx4_tile's order
};

typedef int32_t i32x8 __attribute__((ext_vector_type(8)));

// 16 outputs x 16 rows x 128 inputs; the lowest byte of the exponents counts.
__device__ inline f32x4 mfma_mx4(u32x4 w, uint32_t we, u32x4 x, uint32_t xe, f32x4 c)
{
    const i32x4 a = __builtin_bit_cast(i32x4, w), b = __builtin_bit_cast(i32x4, x);
    const i32x8 a8 = __builtin_shufflevector(a, a, 0, 1, 2, 3, -1, -1, -1, -1), b8 = __builtin_shufflevector(b, b, 0, 1, 2, 3, -1, -1, -1, -1);
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a8, b8, c, 4, 4, 0, (int)we, 0, (int)xe);
}

// Up to 16 NB rows, straight from memory: as k_fused_rows.  VECX: K is a multiple of 32 and rows of
// codes start on 16-byte boundaries; else a block's bytes come one by one.  Bound by latency, by the weights' bytes where these are
// many (7 rows 1536 -> 1536 3.9 us; one row 1536 -> 57,344 10.8 us, 4.4 TB/s).
template <int NB, int MT, int WK, bool VECX>
__global__ __launch_bounds__(64 * WK) void k_mx4_rows(Mx4Args m)
{
    const FusedArgs& a = m.f;
    constexpr int U = VECX ? (MT * NB >= 4 ? 1 : MT * NB >= 2 ? 2 : 4) : 1;  // steps in flight
    const int lane = threadIdx.x % 64, w = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
    const int g = lane / 16, c = lane % 16;
    const int tile0 = blockIdx.x * MT;
    const int64_t b0 = (int64_t)blockIdx.y * 16 * NB;
    const int tiles = fused_tiles<kMx4>(a.n_out), blocks = (a.n_in + kMxBlock - 1) / kMxBlock;
    const uint8_t* const x0 = static_cast<const uint8_t*>(a.x);
    const __amdgpu_buffer_rsrc_t wr = weight_resource(a.P, kBufMaxBytes), er = weight_resource(a.S, kBufMaxBytes);
    static_assert(MT * NB <= WK, "a wave joins one tile's sums");
    OutputColumns<4> columns;
    if (w < MT * NB)
        columns.load(a, fused_output<kMx4>(tile0 + w / NB, g));
    f32x4 acc[MT][NB];
#pragma unroll
    for (int t = 0; t < MT; ++t)
#pragma unroll
        for (int n = 0; n < NB; ++n)
            acc[t][n] = f32x4{};
    for (int s0 = w; s0 < a.steps; s0 += WK * U) {
        u32x4 wt[U][MT], x[U][NB];
        uint32_t we[U][MT], xe[U][NB];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int s = s0 + u * WK;
#pragma unroll
            for (int t = 0; t < MT; ++t) {
                const bool live = s < a.steps && tile0 + t < tiles;
                const uint32_t at = live ? (uint32_t)(tile0 + t) * a.steps + s : 0u;
                wt[u][t] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(wr, live ? lane * 16u : kOutOfRange, at * 1024u, 0));
                we[u][t] = __builtin_amdgcn_raw_buffer_load_b8(er, live ? c * 4u + g : kOutOfRange, at * 64u, 0);
            }
#pragma unroll
            for (int n = 0; n < NB; ++n) {
                // (blocks and rows that are not there are loaded from ones that are, and count as zeros)
                const int64_t b = min(b0 + 16 * n + c, (int64_t)a.B - 1);
                const int block = min(4 * s + g, blocks - 1);
                const uint8_t* const row = x0 + b * a.ld_x;
                if constexpr (VECX) {
                    x[u][n] = *reinterpret_cast<const u32x4*>(row + (int64_t)block * 16);
                } else {
                    uint32_t v[4];
                    mx_row_in(row, block, a.n_in, v);
                    x[u][n] = u32x4{v[0], v[1], v[2], v[3]};
                }
                xe[u][n] = m.scales[b * m.ld_scales + block];
                if (4 * s + g >= blocks)
                    x[u][n] = u32x4{}, xe[u][n] = 127;
            }
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (s0 + u * WK >= a.steps)
                break;
#pragma unroll
            for (int n = 0; n < NB; ++n)
#pragma unroll
                for (int t = 0; t < MT; ++t)
                    acc[t][n] = mfma_mx4(wt[u][t], we[u][t], x[u][n], xe[u][n], acc[t][n]);
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

// Copies rows of any length and alignment for k_mx4_tile: `blocks` (a multiple of 4) blocks of 16 bytes and
// their exponents a row, zeros past K.  A thread a block.
__global__ __launch_bounds__(256) void k_mx4_align(const uint8_t* codes, int64_t ld_codes, const uint8_t* scales, int64_t ld_scales,
                                                   int B, int K, int blocks, uint8_t* out, uint8_t* out_scales)
{
    const int64_t total = (int64_t)B * blocks;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < total; i += (int64_t)gridDim.x * 256) {
        const int64_t b = i / blocks, block = i % blocks;
        const bool live = block * kMxBlock < K;
        uint32_t w[4] = {};
        if (live)
            mx_row_in(codes + b * ld_codes, block, K, w);
        *reinterpret_cast<u32x4*>(out + i * 16) = u32x4{w[0], w[1], w[2], w[3]};
        out_scales[i] = live ? scales[b * ld_scales + block] : 127;
    }
}

// A read of 16 bytes a lane takes 16 lanes at a time: rows 0 to 3 and 12 to 15 of one group of lanes with rows 4 to 11 of the
// next, and the others.  This order gives each of them a place of its own among the 256 bytes that lie in different banks
// (r / 4 % 4 itself: 4.7 million cycles of conflicts in 16,384 rows of 1536 -> 6144; the time was the same).
__device__ inline int mx4_turn(int r) { return -(r / 4) & 3; }

template <int NT, int WM, int WN>
constexpr int mx4_stage_bytes() { return 16 * NT * WN * 64 + WM * WN * 256; }

template <int MT, int NT, int WM, int WN, int D>
constexpr int mx4_tile_lds()
{
    constexpr int ring = D * mx4_stage_bytes<NT, WM, WN>(), turning = WM * WN * 2 * 16 * 16 * MT * 4;
    return ring > turning ? ring : turning;
}

// 16 MT WM outputs x 16 NT WN rows per workgroup of WM x WN waves, 128 inputs a step.  The rows' codes (64 bytes a
// row; chunk q of row r at q ^ mx4_turn(r), so that what is read at a time falls into different banks) and their exponents come
// through a ring of D stages in LDS that loads fill without registers; a wave's weights are its own, so they go
// straight to registers, two steps ahead, each register refilled as soon as its products are issued.
// Bound by the latency of those loads, which one step in flight does not cover, and by the outputs: 16,384 rows 6144 -> 1536 100 us, 3.1
// PFLOP/s (79 without any load, 44 at the rate that these instructions reach from registers), 1536 -> 6144 125, with GELU 152 to 165.
// Slower or no faster: weights through LDS too (107), four and five stages, priorities by workgroup.
// Rows: codes at 16-byte, exponents at 4-byte boundaries, K in whole steps.
template <int MT, int NT, int WM, int WN, int D>
__global__ __launch_bounds__(64 * WM * WN, 2) void k_mx4_tile(Mx4Args m)
{
    const FusedArgs& a = m.f;
    constexpr int kThreads = 64 * WM * WN, kRows = 16 * NT * WN, kWaves = WM * WN;
    constexpr int kChunks = kRows * 4 / kThreads;       // 16-byte chunks of rows that a thread fetches per step
    constexpr int kOwnRows = kRows / kWaves;            // rows whose exponents a wave fetches
    constexpr int kStage = mx4_stage_bytes<NT, WM, WN>();
    constexpr int kExponents = kRows * 64;              // where they begin in a stage
    static_assert(kChunks >= 1 && kRows * 4 % kThreads == 0, "every thread fetches whole chunks");
    static_assert(kOwnRows >= 1 && kOwnRows <= 64 && MT <= 4 && NT % 2 == 0 && D >= 3, "what a load covers");
    extern __shared__ u32x4 s_fused[];
    const int plane_tiles = a.out_tiles * a.row_tiles, total = plane_tiles * a.splits, per_xcd = (total + 7) / 8;
    const int place = (int)(blockIdx.x % 8) * per_xcd + blockIdx.x / 8;
    if ((int)(blockIdx.x / 8) >= per_xcd || place >= total)
        return;
    const int split = place / plane_tiles, id = place % plane_tiles;
    const int group = id / (8 * a.row_tiles), in_group = min(8, a.out_tiles - group * 8);
    const int out_tile = group * 8 + id % (8 * a.row_tiles) % in_group;
    const int row_tile = id % (8 * a.row_tiles) / in_group;
    const int lane = threadIdx.x % 64, w = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
    const int g = lane / 16, c = lane % 16, wm = w % WM, wn = w / WM;
    const int first = split * a.split_steps, steps = min(a.split_steps, a.steps - first);
    const int tiles = fused_tiles<kMx4>(a.n_out);
    const int tile0 = (out_tile * WM + wm) * MT;
    const int64_t b0 = (int64_t)row_tile * kRows;

    const __amdgpu_buffer_rsrc_t wr = weight_resource(a.P, kBufMaxBytes), er = weight_resource(m.E, kBufMaxBytes);
    const __amdgpu_buffer_rsrc_t xr = weight_resource(static_cast<const int8_t*>(a.x) + b0 * a.ld_x, kBufMaxBytes);
    const __amdgpu_buffer_rsrc_t sr = weight_resource(reinterpret_cast<const int8_t*>(m.scales) + b0 * m.ld_scales, kBufMaxBytes);
    const uint32_t fours = (a.steps + 3) / 4;
    uint32_t tile_at[MT], e_at[MT], x_off[kChunks];
#pragma unroll
    for (int t = 0; t < MT; ++t) {  // tiles past the outputs repeat the last one; their results are not stored
        tile_at[t] = (uint32_t)min(tile0 + t, tiles - 1) * a.steps + first;
        e_at[t] = (uint32_t)min(tile0 + t, tiles - 1) * fours;
    }
    const int last_row = (int)min((int64_t)kRows, a.B - b0) - 1;
#pragma unroll
    for (int i = 0; i < kChunks; ++i) {
        const int r = i * (kThreads / 4) + threadIdx.x / 4, q = threadIdx.x % 4 ^ mx4_turn(r);
        x_off[i] = (uint32_t)(min(r, last_row) * a.ld_x) + q * 16u;
    }
    const uint32_t s_off = (uint32_t)(min(w * kOwnRows + min(lane, kOwnRows - 1), last_row) * m.ld_scales);
    const uint32_t lds = lds_address(s_fused);
    // Step s of this workgroup's to stage `buf`; past the last, the last again.
    auto fetch = [&](int buf, int s) __attribute__((always_inline)) {
        const uint32_t at = first + min(s, steps - 1), to = lds + buf * kStage;
        load_words_to_lds(sr, s_off, at * 4u, to + kExponents + w * 256);
#pragma unroll
        for (int i = 0; i < kChunks; ++i)
            load_to_lds(xr, x_off[i], at * 64u, to + (i * (kThreads / 4) + w * 16) * 64);
    };
    u32x4 wt[2][MT];
    uint32_t we[2][MT];
    constexpr int kWeightLoads = 2 * MT;
    auto weights = [&](auto parity, int t, int s) __attribute__((always_inline)) {
        constexpr int q = decltype(parity)::value;
        // (past the last step: zeros)
        const bool live = s < steps;
        const uint32_t at = live ? s : 0;
        wt[q][t] = __builtin_bit_cast(
            u32x4, __builtin_amdgcn_raw_buffer_load_b128(wr, live ? lane * 16u : kOutOfRange, (tile_at[t] + at) * 1024u, 0));
        we[q][t] = __builtin_amdgcn_raw_buffer_load_b32(er, live ? lane * 4u : kOutOfRange, (e_at[t] + (first + at) / 4) * 256u, 0);
    };
    f32x4 acc[MT][NT];
#pragma unroll
    for (int t = 0; t < MT; ++t)
#pragma unroll
        for (int n = 0; n < NT; ++n)
            acc[t][n] = f32x4{};
    // (in the order in which a step asks: rows of D - 1 steps ahead, then weights of two ahead)
#pragma unroll
    for (int s = 0; s < D - 1; ++s) {
        fetch(s, s);
#pragma unroll
        for (int t = 0; t < MT; ++t) {
            if (s == D - 3)
                weights(std::integral_constant<int, 0>{}, t, 0);
            if (s == D - 2)
                weights(std::integral_constant<int, 1>{}, t, 1);
        }
    }
    int cur = 0;
    const char* const ring = reinterpret_cast<const char*>(s_fused);
    auto step = [&](auto parity, int s) __attribute__((always_inline)) {
        constexpr int p = decltype(parity)::value;
        // all but the newest weights have landed for this wave, this stage's rows among it, then for all; and all are done with the stage before it
        wait_loads<kWeightLoads>();
        __syncthreads();
        const char* const stage = ring + cur * kStage;
        u32x4 x[NT];
        uint32_t xe[NT];
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            const int r = (wn * NT + n) * 16 + c;
            x[n] = *reinterpret_cast<const u32x4*>(stage + r * 64 + (g ^ mx4_turn(c)) * 16);
            xe[n] = *reinterpret_cast<const uint32_t*>(stage + kExponents + r / kOwnRows * 256 + r % kOwnRows * 4);
        }
        fetch(cur == 0 ? D - 1 : cur - 1, s + D - 1);
        __builtin_amdgcn_sched_barrier(0);
        uint32_t e[MT];
#pragma unroll
        for (int t = 0; t < MT; ++t)
            e[t] = we[p][t] >> ((first + s) % 4 * 8);
#pragma unroll
        for (int n = 0; n < NT; ++n)
            xe[n] >>= 8 * g;
        // tile by tile, its weights of two steps ahead behind its products
#pragma unroll
        for (int t = 0; t < MT; ++t) {
#pragma unroll
            for (int n = 0; n < NT; ++n)
                acc[t][n] = mfma_mx4(wt[p][t], e[t], x[n], xe[n], acc[t][n]);
            __builtin_amdgcn_sched_barrier(0);
            weights(parity, t, s + 2);
            __builtin_amdgcn_sched_barrier(0);
        }
        cur = cur + 1 == D ? 0 : cur + 1;
    };
    for (int s = 0; s < steps; s += 2) {  // (a step past the last multiplies zeros)
        step(std::integral_constant<int, 0>{}, s);
        step(std::integral_constant<int, 1>{}, s + 1);
    }
    // what was fetched past the last step has landed everywhere before LDS is used anew
    wait_loads<0>();
    __syncthreads();
    const int64_t row0 = b0 + wn * NT * 16, y_at = split * a.split_stride;
    if constexpr (MT % 2 == 0) {
        if (straight_tile<MT>(a, tile0))
            return put_tile_straight<MT, NT, false>(a, acc, tile0, row0, y_at);
    }
    put_tile<MT, NT, false, true>(a, acc, reinterpret_cast<f32x4*>(s_fused) + w * 2 * 16 * 4 * MT, tile0, row0, y_at);
}

}  // namespace spk
