// Host helpers shared by the entry points.
#pragma once
#include <cuda_runtime.h>

#include <atomic>

#include "../../include/apollo.h"

namespace apollo {

// Number of SMs of the current device (asked for once per device: the query costs as much as a small launch).
inline int device_sms(int* sms)
{
    static std::atomic<int> known[64];
    int device = 0;
    if (cudaGetDevice(&device) != cudaSuccess) {
        cudaGetLastError();
        return APOLLO_ERR_CUDA;
    }
    const bool keep = device >= 0 && device < 64;
    int n = keep ? known[device].load(std::memory_order_relaxed) : 0;
    if (n == 0) {
        if (cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, device) != cudaSuccess) {
            cudaGetLastError();
            return APOLLO_ERR_CUDA;
        }
        if (keep) known[device].store(n, std::memory_order_relaxed);
    }
    *sms = n;
    return APOLLO_OK;
}

// Launch whose blocks may start while the launch before it in the stream is still ending (they wait for it themselves:
// ptx::grid_wait_previous).
template <typename... P, typename... A>
cudaError_t launch_after(void (*kernel)(P...), dim3 grid, dim3 block, cudaStream_t stream, A&&... args)
{
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = block;
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, kernel, P(args)...);
}

}  // namespace apollo
