// What the calls without a context (layer norm, rotary positions, gated feed-forward) share on the host.
#pragma once
#include "../../include/hf.h"
#include <cuda.h>
#include <cuda_runtime.h>
#include <stdint.h>

namespace hf_layers {

// What is known of a device after its first call.
struct Device {
    int index, sm_count;
    int* status;            // device status word of the calls without a context, as a context's: [0] flags, [1] detail
    void* encode_tiled;     // cuTensorMapEncodeTiled
    mutable volatile int pairs;     // clusters of two thread blocks with a multiprocessor each that run at a time (0: not asked yet)
};

hf_status fail(hf_status s, const char* fmt, ...);
hf_status current_device(const Device** out);

inline int element_bytes(int type) { return type == HF_F32 ? 4 : 2; }
inline bool aligned(const void* p, size_t bytes) { return (reinterpret_cast<uintptr_t>(p) & (bytes - 1)) == 0; }

// Raises a kernel's limit of dynamic shared memory, once a device (KERNEL: the key, a type of the caller's that stands for the instantiation).
template <typename KERNEL, typename F>
hf_status allow_shared(const Device* d, F kernel, int bytes) {
    static volatile bool done[64];
    if (done[d->index]) return HF_OK;
    const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes);
    if (e != cudaSuccess) return fail(HF_ERR_CUDA, "cudaFuncSetAttribute: %s", cudaGetErrorString(e));
    done[d->index] = true;
    return HF_OK;
}

// Launch of a kernel that may start while the one before it in the stream still runs (it calls pdl_wait() before it touches what that
// kernel wrote).
template <typename... P, typename... A>
hf_status launch_after(void (*kernel)(P...), dim3 grid, dim3 block, size_t smem, cudaStream_t st, A... args) {
    cudaLaunchConfig_t cfg = {};
    cudaLaunchAttribute attr;
    attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr.val.programmaticStreamSerializationAllowed = 1;
    cfg.gridDim = grid; cfg.blockDim = block; cfg.dynamicSmemBytes = smem; cfg.stream = st;
    cfg.attrs = &attr; cfg.numAttrs = 1;
    const cudaError_t e = cudaLaunchKernelEx(&cfg, kernel, args...);
    return e == cudaSuccess ? HF_OK : fail(HF_ERR_CUDA, "cudaLaunchKernelEx: %s", cudaGetErrorString(e));
}

}  // namespace hf_layers

#define HFL_TRY(expr) do { hf_status s_ = (expr); if (s_ != HF_OK) return s_; } while (0)
#define HFL_CUDA(call)                                                                                              \
    do {                                                                                                            \
        cudaError_t e_ = (call);                                                                                    \
        if (e_ != cudaSuccess) return hf_layers::fail(HF_ERR_CUDA, "%s: %s", #call, cudaGetErrorString(e_));         \
    } while (0)
