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

// The runtime keeps an error until it is asked for: taken here, so that the next launch, of this library or of
// anybody else in the process, does not find it.
#define WG_CUDA(expr)                                   \
    do {                                                \
        cudaError_t e__ = (expr);                       \
        if (e__ != cudaSuccess) {                       \
            g_last_cuda_error = (int32_t)e__;           \
            cudaGetLastError();                         \
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

// Sets a kernel's attribute for the current device, the first time only (the call costs the host more than
// half a microsecond).  `done`: of this kernel and attribute, a bit per device.
template <typename Kernel>
cudaError_t set_once(std::atomic<uint64_t> &done, Kernel kernel, cudaFuncAttribute attr, int value) {
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    const uint64_t bit = dev < 64 ? 1ull << dev : 0ull;
    if (done.load(std::memory_order_relaxed) & bit) return cudaSuccess;
    e = cudaFuncSetAttribute(kernel, attr, value);
    if (e == cudaSuccess) done.fetch_or(bit, std::memory_order_relaxed);
    return e;
}

// `groups` clusters of `cluster` blocks.
template <typename... KArgs, typename... Args>
cudaError_t launch_cluster(void (*kernel)(KArgs...), unsigned cluster, unsigned groups, unsigned block, size_t smem,
                           cudaStream_t st, Args... args) {
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = cluster;
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(cluster, groups);
    cfg.blockDim = dim3(block);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    cfg.attrs = attr;
    cfg.numAttrs = 2;
    return cudaLaunchKernelEx(&cfg, kernel, static_cast<KArgs>(args)...);
}

template <typename T>
int32_t dev_alloc(T **p, size_t n) {
    *p = nullptr;
    WG_CUDA(cudaMalloc((void **)p, (n ? n : 1) * sizeof(T)));
    return WG_OK;
}
