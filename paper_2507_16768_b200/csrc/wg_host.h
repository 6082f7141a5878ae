// Host-side helpers shared by the translation units that launch kernels.
#pragma once

#include <atomic>
#include <cstdint>

#include <cuda_runtime.h>
#include <nvtx3/nvToolsExt.h>

#include "wg.h"

// NVTX range around an entry point, so that a timeline shows the calls by name (costs a few
// nanoseconds when no profiler is attached).
struct NvtxRange {
    explicit NvtxRange(const char *name) { nvtxRangePushA(name); }
    ~NvtxRange() { nvtxRangePop(); }
};

inline thread_local int32_t g_last_cuda_error = 0;
inline std::atomic<int64_t> g_launches{0};

#define WG_CUDA(expr)                                   \
    do {                                                \
        cudaError_t e__ = (expr);                       \
        if (e__ != cudaSuccess) {                       \
            g_last_cuda_error = (int32_t)e__;           \
            return WG_ERR_CUDA;                         \
        }                                               \
    } while (0)

// after a <<< >>> launch: count it and pick up a launch-configuration error
#define WG_LAUNCHED()                                   \
    do {                                                \
        g_launches.fetch_add(1, std::memory_order_relaxed); \
        WG_CUDA(cudaGetLastError());                    \
    } while (0)

inline int g_sm_count = 0;
inline int sm_count() {
    if (g_sm_count == 0) {
        int dev = 0, n = 0;
        if (cudaGetDevice(&dev) == cudaSuccess &&
            cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev) == cudaSuccess && n > 0)
            g_sm_count = n;
        else
            g_sm_count = 148;
    }
    return g_sm_count;
}

// Launch with programmatic stream serialization: the kernel may be scheduled while the
// kernel before it in the stream is still running; it orders itself with griddepcontrol.wait.
template <typename... KArgs, typename... Args>
cudaError_t launch_pdl_smem(void (*kernel)(KArgs...), dim3 grid, dim3 block, size_t smem,
                            cudaStream_t st, Args... args) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = block;
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, kernel, static_cast<KArgs>(args)...);
}

template <typename... KArgs, typename... Args>
cudaError_t launch_pdl(void (*kernel)(KArgs...), dim3 grid, dim3 block, cudaStream_t st,
                       Args... args) {
    return launch_pdl_smem(kernel, grid, block, 0, st, args...);
}

template <typename T>
int32_t dev_alloc(T **p, size_t n) {
    *p = nullptr;
    WG_CUDA(cudaMalloc((void **)p, (n ? n : 1) * sizeof(T)));
    return WG_OK;
}
