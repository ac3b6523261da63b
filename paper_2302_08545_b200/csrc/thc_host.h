// What the source files of the C ABI share on the host: errors, dependent launches, a view of the context.
#pragma once
#include "../../include/thc.h"
#include "thc_device.cuh"

#include <string.h>

namespace thc {

// Remembers the error for thc_strerror(); returns THC_ECUDA.
int cuda_fail(cudaError_t e);

#define THC_CUDA(...)                                         \
    do {                                                      \
        cudaError_t e__ = (__VA_ARGS__);                      \
        if (e__ != cudaSuccess) return thc::cuda_fail(e__);   \
    } while (0)

// What calls outside thc.cu need of a context.
struct CtxView {
    DeviceBlock *dev;
    int device;                 // -1: no CUDA device, host-only context
    int sm_count;
    uint32_t in_dtype;
    uint32_t log2_block;
    double t_p;
};
CtxView view_of(const thc_ctx *ctx);

// Whether the context can launch on the current device (THC_OK, THC_EINVAL, THC_ECUDA).
int check_launch_ctx(const thc_ctx *ctx);

// Lets a kernel use more than the default 48 KB of dynamic shared memory (up to 120 KB).
int ensure_dynamic_smem(const void *kern);

inline bool aligned16(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

// A launch that may start while the one before it on the stream is still running (depend_on_previous):
// 1 to 1.5 us less between two launches of a round.
template <class... P, class... A>
cudaError_t launch_after(void (*kern)(P...), dim3 grid, unsigned threads, size_t smem, cudaStream_t st, A... args)
{
    cudaLaunchAttribute attr;
    attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr.val.programmaticStreamSerializationAllowed = 1;
    cudaLaunchConfig_t cfg;
    memset(&cfg, 0, sizeof cfg);
    cfg.gridDim = grid;
    cfg.blockDim = dim3(threads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    cfg.attrs = &attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, kern, P(args)...);
}

}  // namespace thc
