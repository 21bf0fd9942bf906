// Host-side helpers shared by the translation units that define entry points
// of include/salt.h: the context's error message, device and error word (the
// context itself is private to salt_runtime.cu), NVTX ranges and the streams
// that use an object.
#pragma once

#include <vector>

#include <cuda_runtime.h>
#include <nvtx3/nvToolsExt.h>

#include "salt.h"

namespace salt {

// A named NVTX range around a library call on the host (what a timeline
// tool shows next to the kernels the call enqueues); free when no tool is
// attached.
struct NvtxRange {
    explicit NvtxRange(const char *name) { nvtxRangePushA(name); }
    ~NvtxRange() { nvtxRangePop(); }
    NvtxRange(const NvtxRange &) = delete;
    NvtxRange &operator=(const NvtxRange &) = delete;
};

// Sets the context's error message (printf style) and returns s.
salt_status ctx_fail(salt_ctx *ctx, salt_status s, const char *fmt, ...);
// Makes the context's device current.
bool ctx_select_device(salt_ctx *ctx);
int ctx_device(const salt_ctx *ctx);
// The context's device error word (SALT_DEVERR_* bits).
uint32_t *ctx_error_word(salt_ctx *ctx);
// Whether p is device (or managed) memory.
bool on_device(const void *p);

#define SALT_CUDA_OR_FAIL(ctx, call)                                                                                \
    do {                                                                                                            \
        cudaError_t e_ = (call);                                                                                    \
        if (e_ != cudaSuccess) {                                                                                    \
            cudaGetLastError();                                                                                     \
            return ::salt::ctx_fail((ctx), SALT_ERR_CUDA, "%s failed: %s", #call, cudaGetErrorString(e_));          \
        }                                                                                                           \
    } while (0)

// Launches a kernel that may begin while the stream's last one ends (it waits for that one itself).
template <class... P, class... A>
cudaError_t launch_overlapped(void (*kernel)(P...), unsigned blocks, unsigned threads, size_t shared_bytes, cudaStream_t stream, A &&...args)
{
    cudaLaunchConfig_t cfg = {};
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.gridDim = dim3(blocks, 1, 1);
    cfg.blockDim = dim3(threads, 1, 1);
    cfg.dynamicSmemBytes = shared_bytes;
    cfg.stream = stream;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, kernel, static_cast<P>(args)...);
}

}  // namespace salt
