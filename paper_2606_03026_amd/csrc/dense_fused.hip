// Host side of the fused INT8 projection and its gradient (C ABI in
// include/dense_fused.h): handles, validation, choice of the kernel, launches.
#include "dense_fused.h"

#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstdint>
#include <new>

#include "errors.hpp"
#include "fused.hpp"

struct dense_fused {
    int32_t K = 0, M = 0;
    int device = 0;
    int8_t* P = nullptr;     // rows of Q as outputs; the one allocation, which holds the others too
    int8_t* Pt = nullptr;    // columns of Q as outputs (DENSE_FUSED_BACKWARD)
    float* scale = nullptr;  // [M rounded up to 16], zeros past M
};

namespace {

using spk::aligned_to;
using spk::fail;
using spk::FusedArgs;
using spk::hip_fail;
using spk::is_float_type;
using spk::type_bytes;

__global__ __launch_bounds__(256) void k_copy_scale(const float* __restrict__ from, int n, float* __restrict__ to, int padded)
{
    const int i = blockIdx.x * 256 + threadIdx.x;
    if (i < padded)
        to[i] = i < n ? from[i] : 0.0f;
}

void release(dense_fused* h)
{
    (void)hipFree(h->P);
    delete h;
}

int in_eights(const int8_t* Q, int32_t K) { return aligned_to(Q, 8) && K % 8 == 0; }

hipError_t lay_out(const int8_t* Q, const float* scale, bool backward, dense_fused* h)
{
    const int64_t bytes = spk::fused_packed_bytes(h->M, h->K), bytes_t = spk::fused_packed_bytes(h->K, h->M);
    const int padded = (int)spk::fused_pad(h->M, spk::kFusedTile);
    hipError_t e = hipMalloc(&h->P, (size_t)(bytes + (backward ? bytes_t : 0) + padded * (int64_t)sizeof(float)));
    if (e == hipSuccess)
        e = hipDeviceSynchronize();  // Q may still be in flight on any stream
    if (e != hipSuccess)
        return e;
    h->Pt = backward ? h->P + bytes : nullptr;
    h->scale = reinterpret_cast<float*>(h->P + bytes + (backward ? bytes_t : 0));
    const int eights = in_eights(Q, h->K);
    hipLaunchKernelGGL(spk::k_fused_pack<false>, dim3((unsigned)((bytes / 16 + 255) / 256)), dim3(256), 0, nullptr, Q,
                       h->K, h->M, h->P, bytes / 16, eights);
    if (backward)
        hipLaunchKernelGGL(spk::k_fused_pack<true>, dim3((unsigned)((bytes_t / 16 + 255) / 256)), dim3(256), 0, nullptr,
                           Q, h->K, h->M, h->Pt, bytes_t / 16, eights);
    hipLaunchKernelGGL(k_copy_scale, dim3((unsigned)((padded + 255) / 256)), dim3(256), 0, nullptr, scale, h->M,
                       h->scale, padded);
    if ((e = hipGetLastError()) != hipSuccess)
        return e;
    return hipDeviceSynchronize();
}

int check_device(int want)
{
    int dev = -1;
    if (const hipError_t e = hipGetDevice(&dev); e != hipSuccess)
        return hip_fail(e, "hipGetDevice");
    if (dev != want)
        return fail(SPIKE_EINVAL, "handle was created on device %d but device %d is current", want, dev);
    return SPIKE_OK;
}

constexpr int kCUs = 256;

// Up to here a call reads the activations straight from memory.
constexpr int kFewRows = FUSED_FEW_ROWS;

template <typename OT, int NS, int MT, int NT, int WM, int WN, int D, int KS>
void launch_tile(FusedArgs a, hipStream_t st)
{
    a.out_tiles = (a.n_out + 16 * MT * WM - 1) / (16 * MT * WM);
    a.row_tiles = (a.B + 16 * NT * WN - 1) / (16 * NT * WN);
    const int64_t total = (int64_t)a.out_tiles * a.row_tiles * a.splits;
    constexpr unsigned lds = spk::fused_tile_lds<NS, MT, NT, WM, WN, D, KS>();
    static_assert(64 * WM * WN >= 256, "a workgroup can sum a bias gradient too");
    const int64_t sums = a.bias_sums.dbias ? (a.bias_sums.M + 63) / 64 : 0;
    hipLaunchKernelGGL((spk::k_fused_tile<OT, NS, MT, NT, WM, WN, D, KS>), dim3((unsigned)((total + 7) / 8 * 8 + sums)),
                       dim3(64 * WM * WN * KS), lds, st, a);
}

// A tile shape of k_fused_tile (its outputs and rows, the teams that share its steps)
// and what it takes, in us: `fixed` for a call, and for a step of 64 inputs `alone` where
// a compute unit has one tile, `among` for each where it has several.
struct TileShape {
    int outs, rows, teams;
    float fixed, alone, among;
};

// Measured over 1536 -> 1536, 1536 -> 6144 and 6144 -> 1536 with 33 to 4096 rows: BF16
// and F16 (one plane), FP32 (two).
constexpr TileShape kShapes1[] = {{256, 128, 1, 5.8f, 0.79f, 0.95f}, {128, 128, 1, 4.2f, 0.55f, 0.50f},
                                  {128, 64, 1, 4.5f, 0.32f, 0.34f},  {64, 64, 1, 3.8f, 0.25f, 0.206f},
                                  {128, 64, 2, 5.5f, 0.24f, 0.44f},  {64, 32, 2, 3.9f, 0.14f, 0.156f},
                                  {64, 32, 4, 4.7f, 0.10f, 0.24f}};
constexpr TileShape kShapes2[] = {{256, 64, 1, 8.4f, 0.96f, 0.90f}, {128, 32, 1, 7.1f, 0.36f, 0.32f},
                                  {64, 32, 1, 6.4f, 0.29f, 0.203f}, {64, 32, 2, 7.0f, 0.20f, 0.286f},
                                  {128, 64, 1, 7.7f, 0.74f, 0.46f}};

struct TilePlan {
    int shape, splits;
};

// The shape, and the workgroups that share a tile's steps, with the least estimated
// time: the steps of the tiles that come to one compute unit, and for a split the join
// (a launch, and the FP32 sums written and read at 3.9 MB/us).  What that decides
// between, BF16 without an activation, in us: 1536 -> 1536, 64 rows: 6.8 in tiles of 64 x 32 by
// four teams, 9.6 in 64 x 64, 25 in 256 x 128; 1536 -> 6144, 2500 rows: 112 in 64 x 32, 46 in
// 256 x 128; 6144 -> 1536, 33 rows: 14.6 in one part, 11.6 in four; with 1024 rows 30 by two teams,
// 42 in four parts.
TilePlan tile_plan(int ns, int32_t B, int32_t n_out, int32_t steps)
{
    const TileShape* shapes = ns == 1 ? kShapes1 : kShapes2;
    const int n = ns == 1 ? 7 : 5;
    TilePlan best{0, 1};
    float least = 0.0f;
    for (int i = 0; i < n; ++i)
        for (int splits = 1; splits <= 8 && (splits == 1 || steps / splits >= 8); ++splits) {
            const TileShape& t = shapes[i];
            const int64_t tiles = (((int64_t)n_out + t.outs - 1) / t.outs) * (((int64_t)B + t.rows - 1) / t.rows) * splits;
            const int64_t each = (tiles + kCUs - 1) / kCUs;
            float us = t.fixed + (float)((steps + splits - 1) / splits) * (each == 1 ? t.alone : (float)each * t.among);
            if (splits > 1)
                us += 3.5f + (float)splits * (float)B * (float)n_out * (4.0f / 3.9e6f);
            if ((i == 0 && splits == 1) || us < least)
                least = us, best = TilePlan{i, splits};
        }
    // only parts that have steps
    const int each = (steps + best.splits - 1) / best.splits;
    best.splits = (steps + each - 1) / each;
    return best;
}

// The sums of a split product: rows of n_out rounded up to 8 elements.
int64_t split_bytes(const TilePlan& p, int32_t B, int32_t n_out)
{
    return p.splits > 1 ? p.splits * spk::fused_pad(n_out, 8) * B * 4 : 0;
}

// The product of NS planes of activations; `part`: split_bytes for a split one.
template <typename OT, int NS>
void launch_planes(const FusedArgs& a, float* part, hipStream_t st)
{
    const TilePlan p = tile_plan(NS, a.B, a.n_out, a.w_steps);
    FusedArgs t = a;
    t.splits = p.splits;
    t.split_steps = (a.w_steps + p.splits - 1) / p.splits * (a.steps / a.w_steps);
    if (p.splits > 1) {
        t.y = part, t.y_type = SPIKE_TYPE_F32, t.ld_y = spk::fused_pad(a.n_out, 8), t.split_stride = t.ld_y * a.B;
        t.scale = t.row_scale = t.bias = nullptr, t.act = 0, t.residual = t.pre = nullptr, t.vec_out = 1;
    }
    if constexpr (NS == 1) {
        switch (p.shape) {
        case 0: launch_tile<OT, NS, 4, 8, 4, 1, 2, 1>(t, st); break;
        case 1: launch_tile<OT, NS, 2, 8, 4, 1, 2, 1>(t, st); break;
        case 2: launch_tile<OT, NS, 2, 4, 4, 1, 4, 1>(t, st); break;
        case 3: launch_tile<OT, NS, 1, 4, 4, 1, 4, 1>(t, st); break;
        case 4: launch_tile<OT, NS, 2, 4, 4, 1, 4, 2>(t, st); break;
        case 5: launch_tile<OT, NS, 1, 2, 4, 1, 4, 2>(t, st); break;
        default: launch_tile<OT, NS, 1, 2, 4, 1, 4, 4>(t, st); break;
        }
    } else {
        switch (p.shape) {
        case 0: launch_tile<OT, NS, 4, 4, 4, 1, 2, 1>(t, st); break;
        case 1: launch_tile<OT, NS, 2, 2, 4, 1, 4, 1>(t, st); break;
        case 2: launch_tile<OT, NS, 1, 2, 4, 1, 4, 1>(t, st); break;
        case 3: launch_tile<OT, NS, 1, 2, 4, 1, 4, 2>(t, st); break;
        default: launch_tile<OT, NS, 2, 4, 4, 1, 2, 1>(t, st); break;
        }
    }
    if (p.splits > 1) {
        t = a;
        t.splits = p.splits;
        const int64_t ld = spk::fused_pad(a.n_out, 8);
        hipLaunchKernelGGL(spk::k_fused_join, spk::row_grid(a.B, ld / 8), dim3(256), 0, st, t, part, ld);
    }
}

template <typename XT, int NS, int NB, int MT, bool VECX>
void launch_rows(const FusedArgs& a, hipStream_t st)
{
    constexpr int WK = 8;
    const dim3 grid((unsigned)((a.n_out + 16 * MT - 1) / (16 * MT)), (unsigned)((a.B + 16 * NB - 1) / (16 * NB)));
    hipLaunchKernelGGL((spk::k_fused_rows<XT, NS, NB, MT, WK, VECX>), grid, dim3(64 * WK), 0, st, a);
}

// Few rows.  Tiles of outputs that a workgroup takes together share what it does
// to the activations (the cutting of FP32 ones costs more than a tile's weights),
// and the 17th to 32nd row share the weights: FP32, 1536 -> 6144, one row 6.4 us
// one by one and 5.0 by twos; 1536 -> 57,344 29 and 19 by fours, 16 rows 46 and
// 20.  Fewer outputs than that leave compute units idle.
template <typename XT, int NS, bool VECX>
void launch_few(const FusedArgs& a, hipStream_t st)
{
    const int tiles = (a.n_out + 15) / 16;
    if (tiles < kCUs)
        launch_rows<XT, NS, 1, 1, VECX>(a, st);
    else if (tiles < 8 * kCUs)
        launch_rows<XT, NS, 1, 2, VECX>(a, st);
    else if (a.B <= 16)
        launch_rows<XT, NS, 1, 4, VECX>(a, st);
    else
        launch_rows<XT, NS, 2, 4, VECX>(a, st);
}

// Whether the rows of p start on 16-byte boundaries.
bool whole(const void* p, int type, int64_t ld) { return !p || (aligned_to(p, 16) && ld * type_bytes(type) % 16 == 0); }

// Rows that go in groups of 8, 256 of them within a buffer resource.
bool in_chunks(const void* x, int type, int64_t ld, int32_t n)
{
    return whole(x, type, ld) && n % 8 == 0 && ld < spk::kBufMaxBytes / (256 * (int64_t)type_bytes(type));
}

template <typename XT, int NS>
void few_rows(const FusedArgs& a, bool chunks, hipStream_t st)
{
    chunks ? launch_few<XT, NS, true>(a, st) : launch_few<XT, NS, false>(a, st);
}

// Planes of cut activations or gradients: their rows are padded to whole chunks.
int64_t plane_stride(int32_t n) { return spk::fused_pad(n, 8); }
int64_t planes_bytes(int ns, int32_t B, int32_t n) { return spk::fused_pad(ns * plane_stride(n) * B * 2, 16); }

// What forward prepares x into: FP32 rows into two F16 planes and their scales; rows of
// 16-bit elements that do not go in chunks into ones that do.
int64_t prepared_bytes(int x_type, bool chunks, int32_t B, int32_t n)
{
    if (x_type == SPIKE_TYPE_F32)
        return planes_bytes(2, B, n) + spk::fused_pad((int64_t)B * 4, 16);
    return chunks ? 0 : planes_bytes(1, B, n);
}

void cut_rows(FusedArgs& a, void* workspace, hipStream_t st)
{
    const int64_t ld = plane_stride(a.n_in);
    float* undo = reinterpret_cast<float*>(static_cast<char*>(workspace) + planes_bytes(2, a.B, a.n_in));
    hipLaunchKernelGGL(spk::k_fused_cut, dim3((unsigned)std::min(a.B, 1 << 20)), dim3(256), 0, st,
                       static_cast<const float*>(a.x), a.ld_x, a.B, a.n_in, ld, ld * a.B, static_cast<uint16_t*>(workspace),
                       undo, (int)whole(a.x, SPIKE_TYPE_F32, a.ld_x));
    a.x = workspace, a.ld_x = ld, a.plane = ld * a.B, a.n_in = (int)ld, a.row_scale = undo;
}

void align_rows(FusedArgs& a, void* workspace, hipStream_t st)
{
    const int64_t ld = plane_stride(a.n_in);
    hipLaunchKernelGGL(spk::k_fused_align, spk::row_grid(a.B, ld / 8), dim3(256), 0, st, static_cast<const uint16_t*>(a.x),
                       a.ld_x, a.B, a.n_in, ld, static_cast<uint16_t*>(workspace));
    a.x = workspace, a.ld_x = ld, a.n_in = (int)ld;
}

// Rows of a workgroup of the gate, and the parts the bias gradient comes in.
int gate_rows(int32_t B)
{
    return B <= kFewRows ? 1 : (int)std::max<int64_t>(2, ((int64_t)B + spk::kGateParts - 1) / spk::kGateParts);
}
int gate_parts(int32_t B) { return (B + gate_rows(B) - 1) / gate_rows(B); }

// What g * scale is kept in between the gate and the product: two scaled F16 planes and what
// undoes the scaling, apart or side by side in a row; or FP32 rows where the product takes few
// of them, which it cuts itself.  Side by side (a row's planes are whole steps), a tile of one
// plane walks them one after the other; apart, a tile of two takes them together, which is
// faster where sums are long, outputs many and rows fill the tiles.  BF16, us, side by side and
// apart, M summed over -> K: 6144 -> 1536, 64 rows 23.5 and 23.0, 2500 rows 164 and 126, 8192 rows 357
// and 334; 1536 -> 6144, 500 rows 46 and 31, 16,384 rows 549 and 560; 1280 -> 1536, 2500 rows 49
// and 38.  Otherwise: 6000 -> 72, 500 rows 25 and 28; 6000 -> 520, 2500 rows 85 and 93; 72 -> 4104,
// 500 rows 11 and 13; 456 -> 256, 8192 rows 26 and 31; but 1000 -> 1536, 2500 rows 40 and 32.
enum GateForm { kGateRows, kGateApart, kGateBeside };

GateForm gate_form(const dense_fused* h, int y_type, int32_t B)
{
    if (B <= kFewRows)
        return kGateRows;
    return y_type != SPIKE_TYPE_BF16 || (h->M >= 1280 && h->K >= 1024 && B >= 64) ? kGateApart : kGateBeside;
}
int gate_width(GateForm form, int32_t M) { return (int)spk::fused_pad(M, form == kGateBeside ? spk::kFusedStep : 8); }
int64_t gate_plane_bytes(GateForm form, int32_t B, int32_t M)
{
    return spk::fused_pad((int64_t)gate_width(form, M) * B * 4, 16);  // FP32, or twice 16 bits
}
int64_t gate_bytes(GateForm form, int32_t B, int32_t M)
{
    return gate_plane_bytes(form, B, M) + spk::fused_pad((int64_t)B * 4, 16);
}
// Planes that the product takes at a time.
int gate_planes(GateForm form) { return form == kGateApart ? 2 : 1; }

template <typename T, bool PLANES, bool VEC>
void launch_long_gate(const spk::GateArgs& a, hipStream_t st)
{
    if (PLANES && a.gs)
        hipLaunchKernelGGL((spk::k_fused_gate_top<T, VEC>), dim3((unsigned)a.B), dim3(512), 0, st, a);
    const dim3 grid((unsigned)((a.M + spk::kGateCols - 1) / spk::kGateCols), (unsigned)((a.B + a.rows - 1) / a.rows));
    hipLaunchKernelGGL((spk::k_fused_gate_columns<T, PLANES, VEC>), grid, dim3(256), 0, st, a);
}

// Returns the parts that the bias gradient came in: gate_parts at most.
template <typename T, bool PLANES>
int launch_gate(spk::GateArgs a, bool vec, hipStream_t st)
{
    a.rows = gate_rows(a.B);
    if (!vec || a.M > 8192) {
        a.rows = std::max(a.rows, 16);
        vec ? launch_long_gate<T, PLANES, true>(a, st) : launch_long_gate<T, PLANES, false>(a, st);
    } else {
        a.along = (a.M + 511) / 512 * 64;
        a.groups = std::min(a.rows, std::max(1, 768 / a.along));
        hipLaunchKernelGGL((spk::k_fused_gate<T, PLANES>), dim3((unsigned)gate_parts(a.B)), dim3(a.along * a.groups),
                           (a.groups - 1) * a.along * 32, st, a);
    }
    return (a.B + a.rows - 1) / a.rows;
}

int check_rows(int32_t B, int32_t act, int x_type, int y_type)
{
    if (B < 0 || B > FUSED_MAX_B)
        return fail(SPIKE_EINVAL, "B = %d outside [0, %d]", B, FUSED_MAX_B);
    if (act < DENSE_ACT_NONE || act > DENSE_ACT_SILU)
        return fail(SPIKE_EINVAL, "activation %d is not a DENSE_ACT_ value", act);
    if (!is_float_type(x_type) || !is_float_type(y_type))
        return fail(SPIKE_EINVAL, "types %d and %d must be F32, BF16 or F16", x_type, y_type);
    return SPIKE_OK;
}

}  // namespace

extern "C" {

int dense_fused_create(const int8_t* Q, const float* scale, int32_t K, int32_t M, int32_t flags, dense_fused_t* out_handle)
{
    spk::last_error.clear();
    if (!out_handle)
        return fail(SPIKE_EINVAL, "null output handle");
    *out_handle = nullptr;
    if (!Q || !scale)
        return fail(SPIKE_EINVAL, "null pointer (Q %p, scale %p)", (const void*)Q, (const void*)scale);
    if (!aligned_to(scale, 4))
        return fail(SPIKE_EINVAL, "scale must be 4-byte aligned");
    if (K < 1 || K > FUSED_MAX_DIM || M < 1 || M > FUSED_MAX_DIM)
        return fail(SPIKE_EINVAL, "K = %d, M = %d outside [1, %d]", K, M, FUSED_MAX_DIM);
    // (rows of K or M elements, 256 of them, also stay within a buffer resource)
    if (spk::fused_pad(K, 64) * spk::fused_pad(M, 64) >= ((int64_t)1 << 31))
        return fail(SPIKE_EUNSUPPORTED, "K * M = %lld, each rounded up to 64, reaches 2^31", (long long)K * M);
    if (flags & ~DENSE_FUSED_BACKWARD)
        return fail(SPIKE_EINVAL, "unknown flags 0x%x", flags);
    dense_fused* h = new (std::nothrow) dense_fused;
    if (!h)
        return fail(SPIKE_ENOMEM, "out of host memory");
    h->K = K, h->M = M;
    hipError_t e = hipGetDevice(&h->device);
    if (e == hipSuccess)
        e = lay_out(Q, scale, (flags & DENSE_FUSED_BACKWARD) != 0, h);
    if (e != hipSuccess) {
        (void)hipGetLastError();
        release(h);
        return e == hipErrorOutOfMemory ? fail(SPIKE_ENOMEM, "out of device memory for the weights' layout")
                                        : hip_fail(e, "laying out the weights");
    }
    *out_handle = h;
    return SPIKE_OK;
}

int dense_fused_destroy(dense_fused_t h)
{
    spk::last_error.clear();
    if (!h)
        return SPIKE_OK;
    const hipError_t e = hipDeviceSynchronize();
    release(h);
    return e == hipSuccess ? SPIKE_OK : hip_fail(e, "hipDeviceSynchronize");
}

int64_t dense_fused_forward_workspace_bytes(dense_fused_t h, const void* x, int32_t x_type, int64_t ld_x, int32_t B)
{
    if (!h || B < 0 || B > FUSED_MAX_B || !is_float_type(x_type))
        return -1;
    if (B <= kFewRows)
        return 0;
    const int ns = x_type == SPIKE_TYPE_F32 ? 2 : 1;
    const int64_t sums = split_bytes(tile_plan(ns, B, h->M, (h->K + spk::kFusedStep - 1) / spk::kFusedStep), B, h->M);
    return sums + prepared_bytes(x_type, in_chunks(x, x_type, ld_x, h->K), B, h->K);
}

int dense_fused_forward(dense_fused_t h, const void* x, int32_t x_type, int64_t ld_x, int32_t B, const float* bias,
                        int32_t act, const void* residual, int64_t ld_residual, void* y, int32_t y_type, int64_t ld_y,
                        void* pre, int64_t ld_pre, void* workspace, int64_t workspace_bytes, void* stream)
{
    spk::last_error.clear();
    if (!h)
        return fail(SPIKE_EINVAL, "null handle");
    if (int rc = check_rows(B, act, x_type, y_type))
        return rc;
    if (ld_x < h->K || ld_y < h->M || (residual && ld_residual < h->M) || (pre && ld_pre < h->M))
        return fail(SPIKE_EINVAL, "a row stride is below K = %d or M = %d", h->K, h->M);
    if (B == 0)
        return SPIKE_OK;
    if (!x || !y)
        return fail(SPIKE_EINVAL, "null pointer (x %p, y %p)", x, y);
    if (!aligned_to(x, type_bytes(x_type)) || !aligned_to(y, type_bytes(y_type)) || !aligned_to(bias, 4) ||
        !aligned_to(residual, type_bytes(y_type)) || !aligned_to(pre, type_bytes(y_type)))
        return fail(SPIKE_EINVAL, "a pointer is not aligned to its element");
    const int64_t need = dense_fused_forward_workspace_bytes(h, x, x_type, ld_x, B);
    if (need > 0 && (!workspace || workspace_bytes < need || !aligned_to(workspace, 16)))
        return fail(SPIKE_EINVAL, "workspace of %lld bytes at %p, needs %lld, 16-byte aligned",
                    (long long)workspace_bytes, workspace, (long long)need);
    if (int rc = check_device(h->device))
        return rc;
    FusedArgs a{};
    a.P = h->P, a.n_out = h->M, a.n_in = h->K, a.steps = a.w_steps = (h->K + spk::kFusedStep - 1) / spk::kFusedStep;
    a.x = x, a.ld_x = ld_x, a.B = B, a.scale = h->scale, a.bias = bias, a.act = act;
    a.residual = residual, a.ld_residual = ld_residual, a.y = y, a.y_type = y_type, a.ld_y = ld_y;
    a.pre = pre, a.ld_pre = ld_pre;
    a.vec_out = whole(y, y_type, ld_y) && whole(residual, y_type, ld_residual) && whole(pre, y_type, ld_pre);
    const hipStream_t st = static_cast<hipStream_t>(stream);
    const bool chunks = in_chunks(x, x_type, ld_x, h->K);
    if (B <= kFewRows) {
        switch (x_type) {
        case SPIKE_TYPE_F32: few_rows<float, 3>(a, chunks, st); break;
        case SPIKE_TYPE_BF16: few_rows<spk::bf16, 1>(a, chunks, st); break;
        default: few_rows<spk::f16, 1>(a, chunks, st); break;
        }
    } else {
        // the workspace: x prepared where it has to be, then the sums of a split product
        float* part = reinterpret_cast<float*>(static_cast<char*>(workspace) + prepared_bytes(x_type, chunks, B, h->K));
        if (x_type == SPIKE_TYPE_F32)
            cut_rows(a, workspace, st);
        else if (!chunks)
            align_rows(a, workspace, st);
        switch (x_type) {
        case SPIKE_TYPE_F32: launch_planes<spk::f16, 2>(a, part, st); break;
        case SPIKE_TYPE_BF16: launch_planes<spk::bf16, 1>(a, part, st); break;
        default: launch_planes<spk::f16, 1>(a, part, st); break;
        }
    }
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? SPIKE_OK : hip_fail(e, "fused projection launch");
}

int64_t dense_fused_workspace_bytes(dense_fused_t h, int32_t B, int32_t y_type)
{
    if (!h || B < 0 || B > FUSED_MAX_B || !is_float_type(y_type))
        return -1;
    const GateForm form = gate_form(h, y_type, B);
    const int64_t sums = form == kGateRows ? 0
                                           : split_bytes(tile_plan(gate_planes(form), B, h->K,
                                                                   (h->M + spk::kFusedStep - 1) / spk::kFusedStep),
                                                         B, h->K);
    return gate_bytes(form, B, h->M) + sums + spk::fused_pad((int64_t)gate_parts(B) * h->M * 4, 16);
}

int dense_fused_backward(dense_fused_t h, const void* dy, int32_t y_type, int64_t ld_dy, const void* pre, int64_t ld_pre,
                         int32_t act, int32_t B, void* dx, int32_t x_type, int64_t ld_dx, float* dbias, void* workspace,
                         int64_t workspace_bytes, void* stream)
{
    spk::last_error.clear();
    if (!h)
        return fail(SPIKE_EINVAL, "null handle");
    if (int rc = check_rows(B, act, x_type, y_type))
        return rc;
    if (!dx && !dbias)
        return fail(SPIKE_EINVAL, "neither dx nor dbias is asked for");
    if (dx && !h->Pt)
        return fail(SPIKE_EINVAL, "the handle was created without DENSE_FUSED_BACKWARD");
    if (ld_dy < h->M || (act != DENSE_ACT_NONE && pre && ld_pre < h->M) || (dx && ld_dx < h->K))
        return fail(SPIKE_EINVAL, "a row stride is below K = %d or M = %d", h->K, h->M);
    const hipStream_t st = static_cast<hipStream_t>(stream);
    if (B > 0) {
        if (!dy || !workspace || (act != DENSE_ACT_NONE && !pre))
            return fail(SPIKE_EINVAL, "null pointer (dy %p, pre %p, workspace %p)", dy, pre, workspace);
        if (workspace_bytes < dense_fused_workspace_bytes(h, B, y_type))
            return fail(SPIKE_EINVAL, "workspace of %lld bytes, needs %lld", (long long)workspace_bytes,
                        (long long)dense_fused_workspace_bytes(h, B, y_type));
        if (!aligned_to(workspace, 16))
            return fail(SPIKE_EINVAL, "the workspace must be 16-byte aligned");
    }
    if (!aligned_to(dy, type_bytes(y_type)) || !aligned_to(pre, type_bytes(y_type)) || !aligned_to(dx, type_bytes(x_type)) ||
        !aligned_to(dbias, 4))
        return fail(SPIKE_EINVAL, "a pointer is not aligned to its element");
    if (int rc = check_device(h->device))
        return rc;
    if (act == DENSE_ACT_NONE)
        pre = nullptr;
    const GateForm form = gate_form(h, y_type, B);
    const int width = gate_width(form, h->M);
    int parts = 0;
    float* partial = nullptr;
    float* undo = nullptr;
    if (B > 0) {
        undo = reinterpret_cast<float*>(static_cast<char*>(workspace) + gate_plane_bytes(form, B, h->M));
        if (dbias)
            partial = reinterpret_cast<float*>(static_cast<char*>(workspace) + gate_bytes(form, B, h->M));
        spk::GateArgs g{};
        g.dy = dy, g.ld_dy = ld_dy, g.pre = pre, g.ld_pre = ld_pre, g.act = act, g.B = B, g.M = h->M;
        g.scale = h->scale, g.gs = dx ? workspace : nullptr, g.width = width;
        g.ld_gs = form == kGateBeside ? 2 * width : width, g.plane = form == kGateBeside ? width : (int64_t)width * B;
        g.undo = undo, g.partial = partial;
        const bool vec = whole(dy, y_type, ld_dy) && whole(pre, y_type, ld_pre);
        const bool rows = form == kGateRows;
        switch (y_type) {
        case SPIKE_TYPE_F32: parts = rows ? launch_gate<float, false>(g, vec, st) : launch_gate<float, true>(g, vec, st); break;
        case SPIKE_TYPE_BF16: parts = rows ? launch_gate<spk::bf16, false>(g, vec, st) : launch_gate<spk::bf16, true>(g, vec, st); break;
        default: parts = rows ? launch_gate<spk::f16, false>(g, vec, st) : launch_gate<spk::f16, true>(g, vec, st); break;
        }
    }
    // the bias gradient's parts are summed beside the product of many rows, else by themselves
    const spk::BiasArgs sums{partial, parts, h->M, dbias};
    const bool beside = dx && B > kFewRows;
    if (dbias && !beside)
        hipLaunchKernelGGL(spk::k_fused_bias, dim3((unsigned)((h->M + 63) / 64)), dim3(256), 0, st, sums);
    if (dx && B > 0) {
        FusedArgs a{};
        // the rows of g * scale are padded with zeros, as the weights are
        a.P = h->Pt, a.n_out = h->K, a.w_steps = (h->M + spk::kFusedStep - 1) / spk::kFusedStep;
        a.ld_x = form == kGateBeside ? 2 * width : width, a.n_in = (int)a.ld_x;
        a.steps = form == kGateBeside ? 2 * a.w_steps : a.w_steps;
        a.x = workspace, a.plane = (int64_t)width * B, a.B = B;
        a.y = dx, a.y_type = x_type, a.ld_y = ld_dx;
        a.vec_out = whole(dx, x_type, ld_dx);
        if (beside)
            a.bias_sums = sums;
        if (form != kGateRows)
            a.row_scale = undo;
        // the workspace: g * scale (and its rows' scalings), the parts of the bias gradient, the sums of a split product
        float* part = reinterpret_cast<float*>(static_cast<char*>(workspace) + gate_bytes(form, B, h->M) +
                                               spk::fused_pad((int64_t)gate_parts(B) * h->M * 4, 16));
        switch (form) {
        case kGateRows: few_rows<float, 3>(a, true, st); break;
        case kGateApart: launch_planes<spk::f16, 2>(a, part, st); break;
        case kGateBeside: launch_planes<spk::f16, 1>(a, part, st); break;
        }
    }
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? SPIKE_OK : hip_fail(e, "fused projection gradient launch");
}

}  // extern "C"
