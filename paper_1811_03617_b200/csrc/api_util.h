// What the entry points of the C ABI share: checks of pointers, the return code of a failed CUDA call, the device guard.
#pragma once
#include "gvq_internal.h"

namespace gvq {

inline bool aligned16(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

inline gvq_status cuda_fail(gvq_ctx *ctx, cudaError_t e)
{
    if (ctx) ctx->last_cuda_error = (int)e;
    (void)cudaGetLastError();
    // tmap_slot's refusal to upload tensor maps while the stream is being captured
    return e == cudaErrorStreamCaptureUnsupported ? GVQ_ERR_CAPTURE : GVQ_ERR_CUDA;
}

#define GVQ_CUDA(ctx, call)                                    \
    do {                                                       \
        cudaError_t e__ = (call);                              \
        if (e__ != cudaSuccess) return cuda_fail((ctx), e__);  \
    } while (0)

template <typename T>
gvq_status gather_nodes(const T *const *src, int N, NodePtrs<const T> &dst, bool need_align = true)
{
    if (!src) return GVQ_ERR_NULL;
    if (N < 1 || N > GVQ_MAX_NODES) return GVQ_ERR_SHAPE;
    for (int n = 0; n < GVQ_MAX_NODES; ++n) dst.p[n] = nullptr;
    for (int n = 0; n < N; ++n) {
        if (!src[n]) return GVQ_ERR_NULL;
        if (need_align && !aligned16(src[n])) return GVQ_ERR_ALIGN;
        dst.p[n] = src[n];
    }
    return GVQ_OK;
}

// The tables of a context or a plan, from pageable memory, and zeroed counters: on the device when the call returns.  cudaMemcpy
// alone promises that the source has been read and cudaMemset nothing, and a stream that does not wait for the default one (every
// side stream of torch) would not be ordered behind either.
inline cudaError_t upload(void *dst, const void *src, size_t bytes)
{
    const cudaError_t e = cudaMemcpy(dst, src, bytes, cudaMemcpyHostToDevice);
    return e != cudaSuccess ? e : cudaStreamSynchronize(cudaStreamLegacy);
}
inline cudaError_t clear(void *dst, size_t bytes)
{
    const cudaError_t e = cudaMemset(dst, 0, bytes);
    return e != cudaSuccess ? e : cudaStreamSynchronize(cudaStreamLegacy);
}

// Makes the context's device current, and the caller's again at the end; nothing to do where it is already.
struct DeviceGuard {
    int prev = -1;
    bool ok = false;
    explicit DeviceGuard(int dev)
    {
        if (cudaGetDevice(&prev) != cudaSuccess) return;
        if (prev == dev) { prev = -1; ok = true; }
        else ok = cudaSetDevice(dev) == cudaSuccess;
    }
    ~DeviceGuard()
    {
        if (ok && prev >= 0) cudaSetDevice(prev);
    }
};

}  // namespace gvq
