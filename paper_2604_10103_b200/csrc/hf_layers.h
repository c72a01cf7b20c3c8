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
};

hf_status fail(hf_status s, const char* fmt, ...);
hf_status current_device(const Device** out);
inline int element_bytes(int type) { return type == HF_F32 ? 4 : 2; }
inline bool aligned(const void* p, size_t bytes) { return (reinterpret_cast<uintptr_t>(p) & (bytes - 1)) == 0; }

}  // namespace hf_layers

#define HFL_TRY(expr) do { hf_status s_ = (expr); if (s_ != HF_OK) return s_; } while (0)
#define HFL_CUDA(call)                                                                                              \
    do {                                                                                                            \
        cudaError_t e_ = (call);                                                                                    \
        if (e_ != cudaSuccess) return hf_layers::fail(HF_ERR_CUDA, "%s: %s", #call, cudaGetErrorString(e_));         \
    } while (0)
