// What the tensor-core kernels share: the driver's tensor-map encoder and the bounded waits.
#pragma once
#include <cuda.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "apollo_internal.h"
#include "tc_ptx.cuh"

namespace apollo {

constexpr uint32_t TC_WAIT_CAP = 1u << 20;   // polls before a wait gives up (normal waits are far below 1 ms)

typedef CUresult (*EncodeTiledFn)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*,
                                  const cuuint64_t*, const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave,
                                  CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

inline EncodeTiledFn encode_fn()
{
    static EncodeTiledFn fn = nullptr;
    if (!fn) {
        void* p = nullptr;
        cudaDriverEntryPointQueryResult q;
        if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &p, cudaEnableDefault, &q) == cudaSuccess &&
            q == cudaDriverEntryPointSuccess)
            fn = reinterpret_cast<EncodeTiledFn>(p);
    }
    return fn;
}

// Bounded wait on an mbarrier phase.  On expiry the CTA-wide abort flag and the global
// status word are set; later waits return at once, so the kernel always terminates.
// Bounded wait on an mbarrier phase.  false = this wait, or an earlier one of this CTA, gave up: the
// caller stops issuing work and falls through to the barriers and the drain at the end of the kernel.
// `where` names the wait (role and barrier); the first one of a launch that gives up is kept in the word after
// the status word, for whoever has to find out what stalled.
__device__ __forceinline__ bool wait_phase(uint32_t bar, uint32_t parity, volatile int* abort_flag, int32_t* status,
                                           int where = 0)
{
    if (ptx::mbar_try_wait(bar, parity)) return true;      // the common case costs one poll and no flag read
    if (*abort_flag) return false;
    for (uint32_t i = 0; i < TC_WAIT_CAP; ++i)
        if (ptx::mbar_try_wait(bar, parity)) return true;
    *abort_flag = 1;
    atomicCAS(status + 1, 0, where);
    atomicExch(status, STATUS_TIMEOUT);
    return false;
}

// The same for waits that have slack (an epilogue waiting for its accumulator): sleeps between polls,
// which costs nothing there and saves issue slots, i.e. power, on a board that runs at its power cap.
__device__ __forceinline__ bool wait_phase_idle(uint32_t bar, uint32_t parity, volatile int* abort_flag, int32_t* status,
                                                int where = 0)
{
    if (ptx::mbar_try_wait(bar, parity)) return true;
    if (*abort_flag) return false;
    for (uint32_t i = 0; i < TC_WAIT_CAP; ++i) {
        __nanosleep(200);
        if (ptx::mbar_try_wait(bar, parity)) return true;
    }
    *abort_flag = 1;
    atomicCAS(status + 1, 0, where);
    atomicExch(status, STATUS_TIMEOUT);
    return false;
}

// Bounded wait that neither reads nor sets the abort flag: lets copies and MMAs that are already in
// flight finish before the CTA gives up its shared memory and TMEM.
__device__ __forceinline__ void drain_phase(uint32_t bar, uint32_t parity)
{
    for (uint32_t i = 0; i < TC_WAIT_CAP; ++i)
        if (ptx::mbar_try_wait(bar, parity)) return;
}

// Counters in global memory that CTAs of one launch signal each other through.
__device__ __forceinline__ uint32_t ld_acquire_gpu(const uint32_t* p)
{
    uint32_t v;
    asm volatile("ld.acquire.gpu.global.u32 %0, [%1];" : "=r"(v) : "l"(p) : "memory");
    return v;
}
__device__ __forceinline__ void red_release_gpu_add(uint32_t* p, uint32_t v)
{
    asm volatile("red.release.gpu.global.add.u32 [%0], %1;" ::"l"(p), "r"(v) : "memory");
}

}  // namespace apollo
