// Launches of the attention kernels, one translation unit per type of cache (they take a while to compile).
#pragma once

#include "wg_attend.cuh"
#include "wg_host.h"

constexpr int ATTEND_SHARED_WARPS = ATTEND_WARPS;      // of 16 rows each, where the rows of a group are more than 16

template <typename KV, int DP, int WMS, bool GROUPED>
int32_t launch_attend_as(const CacheDev &c, const AttendArgs &a, int64_t most_units, cudaStream_t st) {
    const auto kernel = attend_kernel<KV, DP, WMS, GROUPED>;
    constexpr int smem = Shape<KV, DP>::SMEM;
    static std::atomic<uint64_t> done{0};
    WG_CUDA(set_once(done, kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, smem));
    if (GROUPED) {
        const int32_t row_blocks = (a.group * a.rows + 16 * WMS - 1) / (16 * WMS);
        WG_CUDA(launch_pdl(attend_plan_kernel, dim3((unsigned)a.n_groups), dim3(ATTEND_THREADS), st, c, a, row_blocks));
        WG_LAUNCHED();
    }
    const int64_t room = (int64_t)sm_count() * Shape<KV, DP>::BLOCKS;
    WG_CUDA(launch_pdl_smem(kernel, dim3((unsigned)(most_units < room ? most_units : room)), dim3(ATTEND_THREADS), smem, st, c, a));
    WG_LAUNCHED();
    return WG_OK;
}

template <typename KV, int DP>
int32_t launch_attend_wide(const CacheDev &c, const AttendArgs &a, int64_t most_units, cudaStream_t st) {
    if (a.group == 1 && a.rows <= 16) return launch_attend_as<KV, DP, 1, false>(c, a, most_units, st);
    if (a.group * a.rows <= 16) return launch_attend_as<KV, DP, 1, true>(c, a, most_units, st);
    return launch_attend_as<KV, DP, ATTEND_SHARED_WARPS, true>(c, a, most_units, st);
}

template <typename KV>
int32_t launch_attend(const CacheDev &c, const AttendArgs &a, int64_t most_units, cudaStream_t st) {
    if (c.head_dim <= 64) return launch_attend_wide<KV, 64>(c, a, most_units, st);
    if (c.head_dim <= 128) return launch_attend_wide<KV, 128>(c, a, most_units, st);
    return launch_attend_wide<KV, 256>(c, a, most_units, st);
}

// most_units: what the tables have room for
int32_t attend_bf16(const CacheDev &c, const AttendArgs &a, int64_t most_units, cudaStream_t st);
int32_t attend_fp16(const CacheDev &c, const AttendArgs &a, int64_t most_units, cudaStream_t st);
int32_t attend_e4m3(const CacheDev &c, const AttendArgs &a, int64_t most_units, cudaStream_t st);
int32_t attend_int8(const CacheDev &c, const AttendArgs &a, int64_t most_units, cudaStream_t st);
