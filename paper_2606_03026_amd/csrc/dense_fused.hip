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
    int8_t* P = nullptr;   // rows of Q as outputs
    int8_t* Pt = nullptr;  // columns of Q as outputs (DENSE_FUSED_BACKWARD)
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
    (void)hipFree(h->Pt);
    (void)hipFree(h->scale);
    delete h;
}

hipError_t lay_out(const int8_t* Q, const float* scale, bool backward, dense_fused* h)
{
    const int64_t bytes = spk::fused_packed_bytes(h->M, h->K), bytes_t = spk::fused_packed_bytes(h->K, h->M);
    const int padded = (int)spk::fused_pad(h->M, spk::kFusedTile);
    hipError_t e = hipMalloc(&h->P, (size_t)bytes);
    if (e == hipSuccess && backward)
        e = hipMalloc(&h->Pt, (size_t)bytes_t);
    if (e == hipSuccess)
        e = hipMalloc(&h->scale, padded * sizeof(float));
    if (e == hipSuccess)
        e = hipDeviceSynchronize();  // Q may still be in flight on any stream
    if (e != hipSuccess)
        return e;
    hipLaunchKernelGGL(spk::k_fused_pack<false>, dim3((unsigned)((bytes / 16 + 255) / 256)), dim3(256), 0, nullptr, Q,
                       h->K, h->M, h->P, bytes / 16);
    if (backward)
        hipLaunchKernelGGL(spk::k_fused_pack<true>, dim3((unsigned)((bytes_t / 16 + 255) / 256)), dim3(256), 0, nullptr,
                           Q, h->K, h->M, h->Pt, bytes_t / 16);
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

template <typename XT, int NS, bool VECX>
void launch_product(FusedArgs a, hipStream_t st)
{
    if (a.B <= 32) {
        constexpr int WK = 8;
        const int tiles = (a.n_out + 15) / 16;
        hipLaunchKernelGGL((spk::k_fused_rows<XT, NS, 1, 1, WK, VECX>), dim3((unsigned)tiles, (unsigned)((a.B + 15) / 16)),
                           dim3(64 * WK), 0, st, a);
        return;
    }
    constexpr int MT = 2, NT = 2, WM = 2, WN = 2;
    a.out_tiles = (a.n_out + 16 * MT * WM - 1) / (16 * MT * WM);
    a.row_tiles = (a.B + 16 * NT * WN - 1) / (16 * NT * WN);
    const int64_t total = (int64_t)a.out_tiles * a.row_tiles;
    hipLaunchKernelGGL((spk::k_fused_tile<XT, NS, MT, NT, WM, WN, VECX>), dim3((unsigned)((total + 7) / 8 * 8)),
                       dim3(64 * WM * WN), 0, st, a);
}

template <typename XT, int NS>
void launch_aligned(const FusedArgs& a, hipStream_t st)
{
    if (aligned_to(a.x, 16) && a.ld_x * sizeof(XT) % 16 == 0)
        launch_product<XT, NS, true>(a, st);
    else
        launch_product<XT, NS, false>(a, st);
}

// Four elements of a row of p at a time (8 bytes of the narrow types, 16 of FP32).
bool fours(const void* p, int type, int64_t ld) { return !p || (aligned_to(p, 4 * type_bytes(type)) && ld % 4 == 0); }

// Rows of g * scale in the workspace: whole vectors, at 16-byte boundaries.
int64_t gate_stride(int32_t M) { return spk::fused_pad(M, 8); }
int gate_bytes(int y_type) { return y_type == SPIKE_TYPE_BF16 ? 2 : 4; }
// Rows of a workgroup of the gate, and the parts the bias gradient comes in: at most 32.
int gate_rows(int32_t B) { return (int)std::max<int64_t>(16, ((int64_t)B + 31) / 32); }
int gate_parts(int32_t B) { return (B + gate_rows(B) - 1) / gate_rows(B); }

template <typename T, typename TG>
void launch_gate(const dense_fused* h, const void* dy, int64_t ld_dy, const void* pre, int64_t ld_pre, int act, int32_t B,
                 TG* gs, float* partial, int y_type, hipStream_t st)
{
    const dim3 grid((unsigned)((h->M + spk::kGateCols - 1) / spk::kGateCols), (unsigned)gate_parts(B));
    auto whole = [&](const void* p, int64_t ld) { return !p || (aligned_to(p, 16) && ld * type_bytes(y_type) % 16 == 0); };
    if (whole(dy, ld_dy) && whole(pre, ld_pre))
        hipLaunchKernelGGL((spk::k_fused_gate<T, TG, true>), grid, dim3(256), 0, st, static_cast<const T*>(dy), ld_dy,
                           static_cast<const T*>(pre), ld_pre, act, B, h->M, gate_rows(B), h->scale, gs, gate_stride(h->M),
                           partial);
    else
        hipLaunchKernelGGL((spk::k_fused_gate<T, TG, false>), grid, dim3(256), 0, st, static_cast<const T*>(dy), ld_dy,
                           static_cast<const T*>(pre), ld_pre, act, B, h->M, gate_rows(B), h->scale, gs, gate_stride(h->M),
                           partial);
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

int dense_fused_forward(dense_fused_t h, const void* x, int32_t x_type, int64_t ld_x, int32_t B, const float* bias,
                        int32_t act, const void* residual, int64_t ld_residual, void* y, int32_t y_type, int64_t ld_y,
                        void* pre, int64_t ld_pre, void* stream)
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
    if (int rc = check_device(h->device))
        return rc;
    FusedArgs a{};
    a.P = h->P, a.n_out = h->M, a.n_in = h->K, a.steps = (h->K + spk::kFusedStep - 1) / spk::kFusedStep;
    a.x = x, a.ld_x = ld_x, a.B = B, a.scale = h->scale, a.bias = bias, a.act = act;
    a.residual = residual, a.ld_residual = ld_residual, a.y = y, a.y_type = y_type, a.ld_y = ld_y;
    a.pre = pre, a.ld_pre = ld_pre;
    a.vec_out = fours(y, y_type, ld_y) && fours(residual, y_type, ld_residual) && fours(pre, y_type, ld_pre);
    const hipStream_t st = static_cast<hipStream_t>(stream);
    switch (x_type) {
    case SPIKE_TYPE_F32: launch_aligned<float, 3>(a, st); break;
    case SPIKE_TYPE_BF16: launch_aligned<spk::bf16, 1>(a, st); break;
    default: launch_aligned<spk::f16, 1>(a, st); break;
    }
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? SPIKE_OK : hip_fail(e, "fused projection launch");
}

int64_t dense_fused_workspace_bytes(dense_fused_t h, int32_t B, int32_t y_type)
{
    if (!h || B < 0 || B > FUSED_MAX_B || !is_float_type(y_type))
        return -1;
    return spk::fused_pad(gate_stride(h->M) * B * gate_bytes(y_type), 16) + (int64_t)gate_parts(B) * h->M * 4;
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
    const int parts = B > 0 ? gate_parts(B) : 0;
    float* partial = nullptr;
    if (B > 0) {
        void* gs = dx ? workspace : nullptr;
        partial = dbias ? reinterpret_cast<float*>(static_cast<char*>(workspace) +
                                                   spk::fused_pad(gate_stride(h->M) * B * gate_bytes(y_type), 16))
                        : nullptr;
        switch (y_type) {
        case SPIKE_TYPE_F32:
            launch_gate<float, float>(h, dy, ld_dy, pre, ld_pre, act, B, static_cast<float*>(gs), partial, y_type, st);
            break;
        case SPIKE_TYPE_BF16:
            launch_gate<spk::bf16, spk::bf16>(h, dy, ld_dy, pre, ld_pre, act, B, static_cast<spk::bf16*>(gs), partial,
                                              y_type, st);
            break;
        default:
            launch_gate<spk::f16, float>(h, dy, ld_dy, pre, ld_pre, act, B, static_cast<float*>(gs), partial, y_type, st);
        }
    }
    if (dbias)
        hipLaunchKernelGGL(spk::k_fused_bias, dim3((unsigned)((h->M + 63) / 64)), dim3(64), 0, st, partial, parts, h->M,
                           dbias);
    if (dx && B > 0) {
        FusedArgs a{};
        a.P = h->Pt, a.n_out = h->K, a.n_in = h->M, a.steps = (h->M + spk::kFusedStep - 1) / spk::kFusedStep;
        a.x = workspace, a.ld_x = gate_stride(h->M), a.B = B;
        a.y = dx, a.y_type = x_type, a.ld_y = ld_dx;
        a.vec_out = fours(dx, x_type, ld_dx);
        switch (y_type) {
        case SPIKE_TYPE_F32: launch_aligned<float, 3>(a, st); break;
        case SPIKE_TYPE_BF16: launch_aligned<spk::bf16, 1>(a, st); break;
        default: launch_aligned<float, 2>(a, st); break;
        }
    }
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? SPIKE_OK : hip_fail(e, "fused projection gradient launch");
}

}  // extern "C"
