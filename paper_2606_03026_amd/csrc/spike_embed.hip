// Host side of the embedding lookup and its gradient (C ABI in
// include/spike_embed.h): validation, choice of the vector width, launches.
#include "spike_embed.h"

#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdint>

#include "embed.hpp"
#include "errors.hpp"

namespace {

using spk::aligned_to;
using spk::fail;
using spk::hip_fail;
using spk::is_float_type;
using spk::type_bytes;

// Of the table's zeros, the bytes written beside the merging, the sums and their
// joining (a smaller table's shares below); the rest goes beside the sorting.  A
// 352 MB table's gradient, in runs of 8 or 16: 2,500 tokens 70 us, with nothing beside
// the joining and 128 MB beside the sorting 71; 16,384 tokens 82 and 85.
constexpr int64_t kFillBesideMerge = 48ll << 20, kFillBesideSums = 160ll << 20, kFillBesideJoin = 32ll << 20;

bool rows_vectorize(const void* p, int type, int64_t ld, int32_t D)
{
    const int b = type_bytes(type);
    return D % 8 == 0 && ld % 8 == 0 && aligned_to(p, (uintptr_t)std::min(16, 8 * b));
}

int check_sizes(int32_t T, int32_t V, int32_t D, int32_t id_type, float scale)
{
    if (T < 0 || T > EMBED_MAX_T)
        return fail(SPIKE_EINVAL, "T = %d outside [0, %d]", T, EMBED_MAX_T);
    if (V < 1 || V > EMBED_MAX_V)
        return fail(SPIKE_EINVAL, "V = %d outside [1, %d]", V, EMBED_MAX_V);
    if (D < 1 || D > EMBED_MAX_D)
        return fail(SPIKE_EINVAL, "D = %d outside [1, %d]", D, EMBED_MAX_D);
    if (id_type != SPIKE_TYPE_I32 && id_type != SPIKE_TYPE_I64)
        return fail(SPIKE_EINVAL, "id type %d is not SPIKE_TYPE_I32 or SPIKE_TYPE_I64", id_type);
    if (!std::isfinite(scale))
        return fail(SPIKE_EINVAL, "scale is not finite");
    return SPIKE_OK;
}

struct Lookup {
    const void* table;
    const float* row_scale;
    int32_t V, D;
    int64_t ld_table;
    const void* ids;
    int32_t T;
    float scale;
    void* out;
    int64_t ld_out;
    hipStream_t st;
};

template <typename TI, typename TO, int VEC, typename ID>
void launch_lookup(const Lookup& a)
{
    constexpr int waves = spk::kEmbedBlock / 64;
    hipLaunchKernelGGL((spk::k_embed<TI, TO, VEC, ID>), dim3((unsigned)((a.T + waves - 1) / waves)),
                       dim3(spk::kEmbedBlock), 0, a.st, static_cast<const TI*>(a.table), a.row_scale, a.V, a.D,
                       a.ld_table, static_cast<const ID*>(a.ids), a.T, a.scale, static_cast<TO*>(a.out), a.ld_out);
}

template <typename TI, typename TO>
void lookup_ids(const Lookup& a, bool vec, bool wide_ids)
{
    if (vec)
        wide_ids ? launch_lookup<TI, TO, 8, int64_t>(a) : launch_lookup<TI, TO, 8, int32_t>(a);
    else
        wide_ids ? launch_lookup<TI, TO, 1, int64_t>(a) : launch_lookup<TI, TO, 1, int32_t>(a);
}

template <typename TI>
void lookup_out(const Lookup& a, int out_type, bool vec, bool wide_ids)
{
    switch (out_type) {
    case SPIKE_TYPE_F32: return lookup_ids<TI, float>(a, vec, wide_ids);
    case SPIKE_TYPE_BF16: return lookup_ids<TI, spk::bf16>(a, vec, wide_ids);
    default: return lookup_ids<TI, spk::f16>(a, vec, wide_ids);
    }
}

// The gradient's workspace: keys and positions sorted by chunk, the same for
// the whole list, and two partial sums per run.
struct GradSpace {
    uint32_t *chunk_keys, *keys;
    int *chunk_order, *order;
    float* partial;
};

int64_t grad_space(int32_t T, int32_t D, void* base, GradSpace* out)
{
    const int64_t list = ((int64_t)T * 4 + 255) / 256 * 256;
    const int64_t runs = ((int64_t)T + spk::kRun - 1) / spk::kRun;
    char* p = static_cast<char*>(base);
    if (out) {
        out->keys = reinterpret_cast<uint32_t*>(p);
        out->order = reinterpret_cast<int*>(p + list);
        out->chunk_keys = reinterpret_cast<uint32_t*>(p + 2 * list);
        out->chunk_order = reinterpret_cast<int*>(p + 3 * list);
        out->partial = reinterpret_cast<float*>(p + 4 * list);
    }
    return 4 * list + runs * 2 * D * (int64_t)sizeof(float);
}

struct Grad {
    const void* grad;
    int64_t ld_grad;
    const void* ids;
    int32_t T, V, D;
    float scale;
    int32_t accumulate;
    void* dtable;
    int64_t ld_table;
    GradSpace ws;
    hipStream_t st;
};

// Columns a lane takes: 16 bytes of the gradients.
template <typename TG>
constexpr int vector_of() { return sizeof(TG) == 4 ? 4 : 8; }

// (a launch that failed is the last one: the next reads what it should have written)
template <typename TG, typename TD, int VEC>
hipError_t launch_grad(const Grad& a, const spk::FillArgs& fill, const spk::FillArgs& with_join)
{
    constexpr int waves = spk::kEmbedBlock / 64;
    const int64_t blocks = (a.D + 64 * VEC - 1) / (64 * VEC);
    const int64_t runs = ((int64_t)a.T + spk::kRun - 1) / spk::kRun;
    const int64_t sum_wgs = (runs * blocks + waves - 1) / waves;
    const int64_t wgs = sum_wgs + spk::fill_wgs(fill);
    if (wgs > 0)
        hipLaunchKernelGGL((spk::k_embed_sum<TG, TD, VEC>), dim3((unsigned)wgs), dim3(spk::kEmbedBlock), 0, a.st,
                           static_cast<const TG*>(a.grad), a.ld_grad, a.ws.keys, a.ws.order, a.T, a.D, (int)sum_wgs,
                           a.scale, a.accumulate, static_cast<TD*>(a.dtable), a.ld_table, a.ws.partial, fill);
    if (const hipError_t e = hipGetLastError(); e != hipSuccess)
        return e;
    if (runs > 1)
        hipLaunchKernelGGL((spk::k_embed_join<TD, VEC>), dim3((unsigned)(sum_wgs + spk::fill_wgs(with_join))),
                           dim3(spk::kEmbedBlock), 0, a.st, a.ws.keys, a.T, a.D, a.scale, a.accumulate,
                           static_cast<TD*>(a.dtable), a.ld_table, a.ws.partial, (int)sum_wgs, with_join);
    return hipGetLastError();
}

template <typename TG>
hipError_t grad_table(const Grad& a, int table_type, bool vec, const spk::FillArgs& fill, const spk::FillArgs& with_join)
{
    constexpr int V = vector_of<TG>();
    switch (table_type) {
    case SPIKE_TYPE_F32: return vec ? launch_grad<TG, float, V>(a, fill, with_join) : launch_grad<TG, float, 1>(a, fill, with_join);
    case SPIKE_TYPE_BF16: return vec ? launch_grad<TG, spk::bf16, V>(a, fill, with_join) : launch_grad<TG, spk::bf16, 1>(a, fill, with_join);
    default: return vec ? launch_grad<TG, spk::f16, V>(a, fill, with_join) : launch_grad<TG, spk::f16, 1>(a, fill, with_join);
    }
}

// Cuts the next `bytes` bytes' worth of rows (whole workgroups' rows) off what is left to zero.
spk::FillArgs take_rows(spk::FillArgs* left, int64_t bytes)
{
    spk::FillArgs f = *left;
    const int64_t rows = bytes / std::max<int64_t>(f.bytes, 1) / spk::kFillRows * spk::kFillRows;
    f.count = (int)std::min<int64_t>(rows, left->count);
    left->first += f.count;
    left->count -= f.count;
    return f;
}

}  // namespace

extern "C" {

int spike_embed_forward(const void* table, int32_t table_type, const float* row_scale, int32_t V, int32_t D,
                        int64_t ld_table, const void* ids, int32_t id_type, int32_t T, float scale, void* out,
                        int32_t out_type, int64_t ld_out, void* stream)
{
    spk::last_error.clear();
    if (int rc = check_sizes(T, V, D, id_type, scale))
        return rc;
    if (!is_float_type(table_type) && table_type != SPIKE_TYPE_I8)
        return fail(SPIKE_EINVAL, "table type %d is not F32, BF16, F16 or I8", table_type);
    if (!is_float_type(out_type))
        return fail(SPIKE_EINVAL, "output type %d is not F32, BF16 or F16", out_type);
    if (ld_table < D || ld_out < D)
        return fail(SPIKE_EINVAL, "row strides %lld and %lld must be at least D = %d", (long long)ld_table,
                    (long long)ld_out, D);
    if ((table_type == SPIKE_TYPE_I8) != (row_scale != nullptr))
        return fail(SPIKE_EINVAL, "row scales come with an I8 table, and only with it");
    if (T == 0)
        return SPIKE_OK;
    if (!table || !ids || !out)
        return fail(SPIKE_EINVAL, "null pointer (table %p, ids %p, out %p)", table, ids, out);
    if (!aligned_to(table, type_bytes(table_type)) || !aligned_to(ids, type_bytes(id_type)) ||
        !aligned_to(out, type_bytes(out_type)) || !aligned_to(row_scale, 4))
        return fail(SPIKE_EINVAL, "a pointer is not aligned to its element");
    const Lookup a{table, row_scale, V, D, ld_table, ids, T, scale, out, ld_out, static_cast<hipStream_t>(stream)};
    const bool vec = rows_vectorize(table, table_type, ld_table, D) && rows_vectorize(out, out_type, ld_out, D);
    const bool wide_ids = id_type == SPIKE_TYPE_I64;
    switch (table_type) {
    case SPIKE_TYPE_F32: lookup_out<float>(a, out_type, vec, wide_ids); break;
    case SPIKE_TYPE_BF16: lookup_out<spk::bf16>(a, out_type, vec, wide_ids); break;
    case SPIKE_TYPE_F16: lookup_out<spk::f16>(a, out_type, vec, wide_ids); break;
    default: lookup_out<int8_t>(a, out_type, vec, wide_ids); break;
    }
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? SPIKE_OK : hip_fail(e, "embedding lookup launch");
}

int64_t spike_embed_workspace_bytes(int32_t T, int32_t D)
{
    if (T < 0 || T > EMBED_MAX_T || D < 1 || D > EMBED_MAX_D || (int64_t)T * D > EMBED_MAX_GRAD)
        return -1;
    return grad_space(T, D, nullptr, nullptr);
}

int spike_embed_backward(const void* grad, int32_t grad_type, int64_t ld_grad, const void* ids, int32_t id_type,
                         int32_t T, int32_t V, int32_t D, float scale, int32_t accumulate, void* dtable,
                         int32_t table_type, int64_t ld_table, void* workspace, int64_t workspace_bytes, void* stream)
{
    spk::last_error.clear();
    if (int rc = check_sizes(T, V, D, id_type, scale))
        return rc;
    if (!is_float_type(grad_type) || !is_float_type(table_type))
        return fail(SPIKE_EINVAL, "gradient type %d and table type %d must be F32, BF16 or F16", grad_type, table_type);
    if (ld_grad < D || ld_table < D)
        return fail(SPIKE_EINVAL, "row strides %lld and %lld must be at least D = %d", (long long)ld_grad,
                    (long long)ld_table, D);
    if (accumulate != 0 && accumulate != 1)
        return fail(SPIKE_EINVAL, "accumulate = %d is not 0 or 1", accumulate);
    if ((int64_t)T * D > EMBED_MAX_GRAD)
        return fail(SPIKE_EUNSUPPORTED, "T * D = %lld exceeds %lld", (long long)T * D, (long long)EMBED_MAX_GRAD);
    if (T == 0 && accumulate)
        return SPIKE_OK;
    if (!dtable || (T > 0 && (!grad || !ids || !workspace)))
        return fail(SPIKE_EINVAL, "null pointer (grad %p, ids %p, dtable %p, workspace %p)", grad, ids, dtable,
                    workspace);
    if (!aligned_to(grad, type_bytes(grad_type)) || !aligned_to(ids, type_bytes(id_type)) ||
        !aligned_to(dtable, type_bytes(table_type)))
        return fail(SPIKE_EINVAL, "a pointer is not aligned to its element");
    if (T > 0 && !aligned_to(workspace, 16))
        return fail(SPIKE_EINVAL, "the workspace must be 16-byte aligned");
    if (workspace_bytes < (T > 0 ? spike_embed_workspace_bytes(T, D) : 0))
        return fail(SPIKE_EINVAL, "workspace of %lld bytes, needs %lld", (long long)workspace_bytes,
                    (long long)spike_embed_workspace_bytes(T, D));
    Grad a{grad, ld_grad, ids, T, V, D, scale, accumulate, dtable, ld_table, {}, static_cast<hipStream_t>(stream)};
    const bool vec = rows_vectorize(grad, grad_type, ld_grad, D) && rows_vectorize(dtable, table_type, ld_table, D);
    const int64_t elem = type_bytes(table_type);
    spk::FillArgs fill{static_cast<char*>(dtable), ld_table * elem, D * elem, 0, accumulate ? 0 : V,
                       (int)rows_vectorize(dtable, table_type, ld_table, D)};
    spk::FillArgs with_join = fill;
    with_join.count = 0;
    if (T > 0) {
        grad_space(T, D, workspace, &a.ws);
        const bool one = T <= spk::kSortChunk;
        const int wgs = (T + spk::kSortTokens - 1) / spk::kSortTokens;
        uint32_t* k = one ? a.ws.keys : a.ws.chunk_keys;
        int* o = one ? a.ws.order : a.ws.chunk_order;
        // Rows zeroed beside the sorting, before it is known which are named (those are
        // then written again); the others go beside the sums and their joining.
        const int64_t all = fill.count * fill.bytes;
        if (T > spk::kRun)
            with_join = take_rows(&fill, std::min<int64_t>(kFillBesideJoin, all / 8));
        const int64_t beside_sums = std::min<int64_t>(kFillBesideSums, all / 2);
        const int64_t beside_merge = one ? 0 : std::min<int64_t>(kFillBesideMerge, all / 8);
        const spk::FillArgs with_sort = take_rows(&fill, fill.count * fill.bytes - beside_sums - beside_merge);
        const dim3 block(spk::kEmbedBlock), grid((unsigned)(wgs + spk::fill_wgs(with_sort)));
        if (id_type == SPIKE_TYPE_I64)
            hipLaunchKernelGGL(spk::k_embed_sort<int64_t>, grid, block, 0, a.st, static_cast<const int64_t*>(ids), T, V,
                               k, o, wgs, with_sort);
        else
            hipLaunchKernelGGL(spk::k_embed_sort<int32_t>, grid, block, 0, a.st, static_cast<const int32_t*>(ids), T, V,
                               k, o, wgs, with_sort);
        if (const hipError_t e = hipGetLastError(); e != hipSuccess)
            return hip_fail(e, "embedding gradient launch");
        if (!one) {
            const spk::FillArgs with_merge = take_rows(&fill, beside_merge);
            hipLaunchKernelGGL(spk::k_embed_merge, dim3((unsigned)(wgs + spk::fill_wgs(with_merge))), block, 0, a.st, k, o,
                               T, a.ws.keys, a.ws.order, wgs, with_merge);
            if (const hipError_t e = hipGetLastError(); e != hipSuccess)
                return hip_fail(e, "embedding gradient launch");
        }
    }
    hipError_t e = hipSuccess;
    switch (grad_type) {
    case SPIKE_TYPE_F32: e = grad_table<float>(a, table_type, vec, fill, with_join); break;
    case SPIKE_TYPE_BF16: e = grad_table<spk::bf16>(a, table_type, vec, fill, with_join); break;
    default: e = grad_table<spk::f16>(a, table_type, vec, fill, with_join); break;
    }
    return e == hipSuccess ? SPIKE_OK : hip_fail(e, "embedding gradient launch");
}

}  // extern "C"
