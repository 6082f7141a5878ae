// Launches of the attention kernels, one translation unit per type of cache (they take a while to compile).
#pragma once

#include "wg_attend.cuh"
#include "wg_host.h"

template <typename KV, int DP, int SHARED_WARPS, bool GROUPED, int NT>
int32_t launch_attend_as(const CacheDev &c, const AttendArgs &a, int64_t most_tiles, cudaStream_t st) {
    const auto kernel = attend_kernel<KV, DP, SHARED_WARPS, GROUPED, NT>;
    constexpr int smem = Shape<KV, DP>::SMEM;
    static std::atomic<uint64_t> done{0};
    WG_CUDA(set_once(done, kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, smem));
    if (GROUPED) {
        WG_CUDA(launch_pdl(attend_plan_kernel, dim3((unsigned)a.n_groups), dim3(ATTEND_THREADS), st, c, a));
        WG_LAUNCHED();
    }
    // (two at least: one for what is shared, one for what is not)
    const int64_t room = (int64_t)sm_count() * Shape<KV, DP>::BLOCKS, blocks = most_tiles < 2 ? 2 : most_tiles < room ? most_tiles : room;
    WG_CUDA(launch_pdl_smem(kernel, dim3((unsigned)blocks), dim3(ATTEND_THREADS), smem, st, c, a));
    WG_LAUNCHED();
    return WG_OK;
}

constexpr int FEW_PAIRS = 128;

template <typename KV, int DP>
int32_t launch_attend_wide(const CacheDev &c, const AttendArgs &a, int64_t most_tiles, cudaStream_t st) {
    if (a.group == 1 && a.rows <= 16) {
        const bool few = (int64_t)a.n_tokens * c.n_heads < FEW_PAIRS;
        if (a.rows <= 8)
            return few ? launch_attend_as<KV, DP, 1, false, 1>(c, a, most_tiles, st) : launch_attend_as<KV, DP, 0, false, 1>(c, a, most_tiles, st);
        return few ? launch_attend_as<KV, DP, 1, false, 2>(c, a, most_tiles, st) : launch_attend_as<KV, DP, 0, false, 2>(c, a, most_tiles, st);
    }
    if (a.rows > 8) return launch_attend_as<KV, DP, ATTEND_WARPS, true, 2>(c, a, most_tiles, st);
    if (a.group * a.rows <= 8) return launch_attend_as<KV, DP, 1, true, 1>(c, a, most_tiles, st);
    return launch_attend_as<KV, DP, ATTEND_WARPS, true, 1>(c, a, most_tiles, st);
}

template <typename KV>
int32_t launch_attend(const CacheDev &c, const AttendArgs &a, int64_t most_tiles, cudaStream_t st) {
    if (c.head_dim <= 64) return launch_attend_wide<KV, 64>(c, a, most_tiles, st);
    if (c.head_dim <= 128) return launch_attend_wide<KV, 128>(c, a, most_tiles, st);
    return launch_attend_wide<KV, 256>(c, a, most_tiles, st);
}

// most_tiles: of 16 positions of a head, what the tables have room for
int32_t attend_bf16(const CacheDev &c, const AttendArgs &a, int64_t most_tiles, cudaStream_t st);
int32_t attend_fp16(const CacheDev &c, const AttendArgs &a, int64_t most_tiles, cudaStream_t st);
int32_t attend_e4m3(const CacheDev &c, const AttendArgs &a, int64_t most_tiles, cudaStream_t st);
int32_t attend_int8(const CacheDev &c, const AttendArgs &a, int64_t most_tiles, cudaStream_t st);
