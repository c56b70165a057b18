// Host side of the gradients' norm and its clipping (C ABI in
// include/spike_clip.h): the table of chunks, validation, two launches.
#include "spike_clip.h"

#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstdint>
#include <new>
#include <vector>

#include "clip.hpp"
#include "errors.hpp"

struct spike_clip {
    int device = 0;
    int64_t chunks = 0;
    spk::ClipChunk* table = nullptr;
};

namespace {

using spk::aligned_to;
using spk::fail;
using spk::hip_fail;

struct Span {
    uintptr_t from, to;
    int32_t tensor;
    bool out;
};

// Whether no output meets another output or another tensor's gradient.
bool apart(std::vector<Span>& spans)
{
    std::sort(spans.begin(), spans.end(), [](const Span& a, const Span& b) { return a.from < b.from; });
    // the furthest end so far, of outputs and of gradients, and of those of another tensor
    struct Far {
        uintptr_t to = 0, other = 0;
        int32_t tensor = -1;
        uintptr_t without(int32_t t) const { return t == tensor ? other : to; }
        void add(const Span& s)
        {
            if (s.tensor == tensor) {
                to = std::max(to, s.to);
            } else if (s.to > to) {
                other = to, to = s.to, tensor = s.tensor;
            } else {
                other = std::max(other, s.to);
            }
        }
    } outs, grads;
    for (const Span& s : spans) {
        if (outs.without(s.tensor) > s.from || (s.out && grads.without(s.tensor) > s.from))
            return false;
        (s.out ? outs : grads).add(s);
    }
    return true;
}

int build(const void* const* grads, void* const* outs, const int32_t* types, const int64_t* sizes, int32_t n,
          std::vector<spk::ClipChunk>& chunks)
{
    std::vector<Span> spans;
    int64_t total = 0;
    for (int32_t i = 0; i < n; ++i) {
        if (!spk::is_float_type(types[i]))
            return fail(SPIKE_EINVAL, "tensor %d: type %d is not F32, BF16 or F16", i, types[i]);
        if (sizes[i] < 0 || sizes[i] > ((int64_t)1 << 40) || (total += sizes[i]) > ((int64_t)1 << 40))
            return fail(SPIKE_EINVAL, "tensor %d: %lld elements, or more than 2^40 up to here", i, (long long)sizes[i]);
        if (sizes[i] == 0)
            continue;
        const int64_t b = spk::type_bytes(types[i]);
        const char* const in = static_cast<const char*>(grads[i]);
        char* const out = outs && outs[i] ? static_cast<char*>(outs[i]) : const_cast<char*>(in);
        if (!in || !aligned_to(in, b) || !aligned_to(out, b))
            return fail(SPIKE_EINVAL, "tensor %d: pointers %p, %p must be set and aligned to their elements", i,
                        (const void*)in, (void*)out);
        const uintptr_t bytes = (uintptr_t)(sizes[i] * b), from = (uintptr_t)in, to = (uintptr_t)out;
        if (in != out && from < to + bytes && to < from + bytes)
            return fail(SPIKE_EINVAL, "tensor %d: the output overlaps its gradient without being it", i);
        if (in != out)
            spans.push_back(Span{from, from + bytes, i, false});
        spans.push_back(Span{to, to + bytes, i, true});
        for (int64_t at = 0; at < sizes[i]; at += spk::kClipChunk)
            chunks.push_back(spk::ClipChunk{in + at * b, out + at * b, (int32_t)std::min<int64_t>(spk::kClipChunk, sizes[i] - at), types[i]});
    }
    if (!apart(spans))
        return fail(SPIKE_EINVAL, "an output overlaps another output or another tensor's gradient");
    return SPIKE_OK;
}

int wgs_of(const spike_clip* h) { return (int)std::min<int64_t>(std::max<int64_t>(h->chunks, 1), spk::kClipWgs); }

}  // namespace

extern "C" {

int spike_clip_create(const void* const* grads, void* const* outs, const int32_t* types, const int64_t* sizes, int32_t n,
                      spike_clip_t* out_handle)
{
    spk::last_error.clear();
    if (!out_handle)
        return fail(SPIKE_EINVAL, "null output handle");
    *out_handle = nullptr;
    if (n < 0 || n > CLIP_MAX_TENSORS)
        return fail(SPIKE_EINVAL, "n = %d outside [0, %d]", n, CLIP_MAX_TENSORS);
    if (n > 0 && (!grads || !types || !sizes))
        return fail(SPIKE_EINVAL, "null array (grads %p, types %p, sizes %p)", (const void*)grads, (const void*)types,
                    (const void*)sizes);
    spike_clip* h = nullptr;
    try {
        std::vector<spk::ClipChunk> chunks;
        if (int rc = build(grads, outs, types, sizes, n, chunks))
            return rc;
        h = new spike_clip;
        h->chunks = (int64_t)chunks.size();
        const size_t bytes = chunks.size() * sizeof(spk::ClipChunk);
        hipError_t e = hipGetDevice(&h->device);
        if (e == hipSuccess && bytes > 0)
            e = hipMalloc(&h->table, bytes);
        if (e == hipSuccess && bytes > 0)
            e = hipMemcpy(h->table, chunks.data(), bytes, hipMemcpyHostToDevice);
        if (e != hipSuccess) {
            (void)hipGetLastError();
            (void)hipFree(h->table);
            delete h;
            return e == hipErrorOutOfMemory ? fail(SPIKE_ENOMEM, "out of device memory for the table of %zu chunks", chunks.size())
                                            : hip_fail(e, "the table of gradients");
        }
    } catch (const std::bad_alloc&) {
        delete h;
        return fail(SPIKE_ENOMEM, "out of host memory");
    }
    *out_handle = h;
    return SPIKE_OK;
}

int spike_clip_destroy(spike_clip_t h)
{
    spk::last_error.clear();
    if (!h)
        return SPIKE_OK;
    const hipError_t e = hipDeviceSynchronize();
    (void)hipFree(h->table);
    delete h;
    return e == hipSuccess ? SPIKE_OK : hip_fail(e, "hipDeviceSynchronize");
}

int64_t spike_clip_workspace_bytes(spike_clip_t h) { return h ? ((int64_t)wgs_of(h) * 8 + 15) / 16 * 16 : -1; }

int spike_clip_forward(spike_clip_t h, float max_norm, float* result, void* workspace, int64_t workspace_bytes, void* stream)
{
    spk::last_error.clear();
    if (!h)
        return fail(SPIKE_EINVAL, "null handle");
    if (!(max_norm > 0.0f))
        return fail(SPIKE_EINVAL, "max_norm = %g must be positive", max_norm);
    if (!result || !aligned_to(result, 4))
        return fail(SPIKE_EINVAL, "result %p must be set and 4-byte aligned", (void*)result);
    const int64_t need = spike_clip_workspace_bytes(h);
    if (!workspace || workspace_bytes < need || !aligned_to(workspace, 16))
        return fail(SPIKE_EINVAL, "workspace of %lld bytes at %p, needs %lld, 16-byte aligned", (long long)workspace_bytes,
                    workspace, (long long)need);
    int dev = -1;
    if (const hipError_t e = hipGetDevice(&dev); e != hipSuccess)
        return hip_fail(e, "hipGetDevice");
    if (dev != h->device)
        return fail(SPIKE_EINVAL, "handle was created on device %d but device %d is current", h->device, dev);
    const hipStream_t st = static_cast<hipStream_t>(stream);
    const spk::ClipArgs a{h->table, h->chunks, static_cast<double*>(workspace), wgs_of(h), max_norm, result};
    hipLaunchKernelGGL(spk::k_clip_squares, dim3(a.wgs), dim3(256), 0, st, a);
    // (the factor comes from the sums: nothing is scaled without them)
    hipError_t e = hipGetLastError();
    if (e == hipSuccess) {
        hipLaunchKernelGGL(spk::k_clip_scale, dim3(a.wgs), dim3(256), 0, st, a);
        e = hipGetLastError();
    }
    return e == hipSuccess ? SPIKE_OK : hip_fail(e, "gradient clipping launch");
}

}  // extern "C"
