// Host-side helpers of the decoder operators: argument checks shared by their C entry points.
#pragma once

#include <cuda_runtime.h>

#include <cmath>
#include <cstdint>
#include <exception>
#include <new>

#include "objects.h"

namespace btc {

inline bool decoder_type(btc_dtype_t t) { return t == BTC_F32 || t == BTC_F16 || t == BTC_BF16; }

inline bool aligned_to(const void *p, size_t bytes) { return reinterpret_cast<uintptr_t>(p) % bytes == 0; }

// Is a number that was given as a double finite as fp32, which the kernels compute in?
inline bool fits_f32(double x) { return std::isfinite(float(x)); }

// |stride| * (extent - 1) summed stays far inside int64: the kernels form offsets without overflow tests
inline bool spans_fit(const TensorDesc &t)
{
    const __int128 limit = __int128(1) << 60;
    __int128 span = 0;
    for (size_t i = 0; i < t.extent.size(); ++i) {
        const __int128 s = t.stride[i] < 0 ? -__int128(t.stride[i]) : __int128(t.stride[i]);
        span += s * (t.extent[i] - 1);
        if (span > limit || s > limit) return false;
    }
    return true;
}

// Runs the body of a C entry point; nothing thrown inside (only allocation can throw) leaves it.
template <typename F> btc_error_t guarded(F &&body)
{
    try {
        return body();
    } catch (const std::bad_alloc &) {
        return BTC_ERR_OUT_OF_MEMORY;
    } catch (const std::exception &) {
        return BTC_ERR_INVALID_ARGUMENT;
    }
}

// One launch that may be set up while the kernel before it in the stream runs (the kernels wait on the device).
template <typename... Args, typename... Given>
btc_error_t launch_early(void (*kernel)(Args...), dim3 blocks, unsigned threads, size_t shared, cudaStream_t st, Given &&...given)
{
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = blocks;
    cfg.blockDim = dim3(threads);
    cfg.dynamicSmemBytes = shared;
    cfg.stream = st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    if (cudaLaunchKernelEx(&cfg, kernel, Args(given)...) != cudaSuccess) {
        cudaGetLastError();
        return BTC_ERR_CUDA;
    }
    return BTC_SUCCESS;
}

}  // namespace btc
