// Launches of the attention kernels, one translation unit per type of cache (they take a while to compile).
#pragma once

#include "wg_attend.cuh"
#include "wg_host.h"

// The kernel that joins what was cut; the same for all types of cache.  head_dim: as the kernels round it.
int32_t attend_join(const CacheDev &c, const AttendArgs &a, int head_dim, cudaStream_t st);

template <typename KV, int DP, int SHARED_WARPS, bool GROUPED, int NTS, int NT>
int32_t launch_attend_as(const CacheDev &c, AttendArgs a, int64_t most_tiles, cudaStream_t st) {
    using S = Shape<KV, DP>;
    const auto kernel = attend_kernel<KV, DP, SHARED_WARPS, GROUPED, NTS, NT>;
    static std::atomic<uint64_t> done{0};
    WG_CUDA(set_once(done, kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)S::SMEM));
    using A = Attend<KV, DP, SHARED_WARPS, GROUPED, NTS, NT>;
    a.grouped = GROUPED, a.origins = S::NARROW, a.warp_rows = A::WARP_ROWS, a.shared_rows_each = A::ROWS;
    a.shared_row_blocks = SHARED_WARPS == 0 ? 0 : GROUPED ? (a.group * a.rows + A::ROWS - 1) / A::ROWS : a.row_blocks;
    if (GROUPED) {
        WG_CUDA(launch_pdl(attend_plan_kernel, dim3((unsigned)a.n_groups), dim3(ATTEND_THREADS), st, c, a));
        WG_LAUNCHED();
    }
    // (two at least: one for what is shared, one for what is not)
    const int64_t room = (int64_t)sm_count() * S::BLOCKS, blocks = most_tiles < 2 ? 2 : most_tiles < room ? most_tiles : room;
    WG_CUDA(launch_pdl_smem(kernel, dim3((unsigned)blocks), dim3(ATTEND_THREADS), S::SMEM, st, c, a));
    WG_LAUNCHED();
    return attend_join(c, a, DP, st);
}


template <typename KV, int DP>
int32_t launch_attend_wide(const CacheDev &c, const AttendArgs &a, int64_t most_tiles, cudaStream_t st) {
    if (a.group == 1 && a.rows <= 16) {
        // Few (token, key head) pairs: a block works on one at a time, its warps side by side.  Many: every warp by itself.  (16-bit
        // caches, 256 pairs of 4096 positions: 74.6 and 75.2 us; 512 of 500: 28.6 and 29.7; 64 of 500: 9.7 and 13.2.  8-bit ones,
        // 128 pairs of 16384: 93 and 83; 64: 46.2 and 45.8.)
        const bool few = (int64_t)a.n_tokens * c.n_heads < (Shape<KV, DP>::NARROW ? 128 : 4 * sm_count());
        if (a.rows <= 8)
            return few ? launch_attend_as<KV, DP, 1, false, 1, 1>(c, a, most_tiles, st) : launch_attend_as<KV, DP, 0, false, 1, 1>(c, a, most_tiles, st);
        return few ? launch_attend_as<KV, DP, 1, false, 2, 2>(c, a, most_tiles, st) : launch_attend_as<KV, DP, 0, false, 2, 2>(c, a, most_tiles, st);
    }
    const int32_t rows = a.group * a.rows;
    if (a.rows > 8) return launch_attend_as<KV, DP, 4, true, 2, 2>(c, a, most_tiles, st);
    if (rows <= 16) return launch_attend_as<KV, DP, 1, true, 2, 1>(c, a, most_tiles, st);
    if (rows <= 32) return launch_attend_as<KV, DP, 2, true, 2, 1>(c, a, most_tiles, st);
    return launch_attend_as<KV, DP, 4, true, 2, 1>(c, a, most_tiles, st);
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
