// Attention over a paged cache (wg_attend_*, wg_kv_attend of wg.h): scratch, checks and launches.
#include <cmath>
#include <new>

#include "wg_attend.h"

struct wg_attend {
    int32_t max_tokens = 0, n_q_heads = 0, n_heads = 0, head_dim = 0;
    int32_t *shared = nullptr;
    int2 *shared_cuts = nullptr, *own_cuts = nullptr;
    float *block_parts = nullptr, *warp_parts = nullptr, *shared_rows = nullptr, *own_rows = nullptr;
};

namespace {

constexpr float LOG2_E = 1.44269504088896f;

// A row of partial results: the head size as the kernels round it, a maximum and a sum.
int64_t part_row(int32_t head_dim) { return (head_dim <= 64 ? 64 : head_dim <= 128 ? 128 : 256) + 4; }

template <int DP, int WARPS>
int32_t launch_join_by(const CacheDev &c, const AttendArgs &a, cudaStream_t st) {
    const dim3 grid((unsigned)((a.n_q_heads * WARPS + ATTEND_WARPS - 1) / ATTEND_WARPS), (unsigned)a.n_tokens);
    const auto kernel = a.origins ? attend_join_kernel<DP, WARPS, true> : attend_join_kernel<DP, WARPS, false>;
    WG_CUDA(launch_pdl(kernel, grid, dim3(ATTEND_THREADS), st, c, a));
    WG_LAUNCHED();
    return WG_OK;
}

// A block per row where there are few rows, or few pairs, which then have many parts each; else a warp.  (32 x 4096 positions, 1024
// rows: 74.8 us with blocks, 76.6 with warps; 128 x 128, 4096 rows: 26.5 and 22.7; 24 x 4 drafted tokens, 96 pairs: 28 and 31.)
template <int DP>
int32_t launch_join(const CacheDev &c, const AttendArgs &a, cudaStream_t st) {
    if ((int64_t)a.n_tokens * a.n_q_heads <= (int64_t)sm_count() * 8 || (int64_t)a.n_groups * c.n_heads <= sm_count())
        return launch_join_by<DP, ATTEND_WARPS>(c, a, st);
    return launch_join_by<DP, 1>(c, a, st);
}

}  // namespace

int32_t attend_join(const CacheDev &c, const AttendArgs &a, int head_dim, cudaStream_t st) {
    return head_dim == 64 ? launch_join<64>(c, a, st) : head_dim == 128 ? launch_join<128>(c, a, st) : launch_join<256>(c, a, st);
}

extern "C" {

int32_t wg_attend_create(int32_t max_tokens, int32_t n_q_heads, int32_t n_heads, int32_t head_dim, wg_attend **out) {
    NvtxRange nvtx_range("wg_attend_create");
    if (!out) return WG_ERR_ARG;
    *out = nullptr;
    if (max_tokens < 1 || n_heads < 1 || n_heads > 1024 || n_q_heads < n_heads || n_q_heads > 65535 || n_q_heads % n_heads ||
        head_dim < 16 || head_dim > WG_KV_MAX_HEAD_DIM || head_dim % 16)
        return WG_ERR_ARG;
    wg_attend *p = new (std::nothrow) wg_attend();
    if (!p) return WG_ERR_ARG;
    p->max_tokens = max_tokens, p->n_q_heads = n_q_heads, p->n_heads = n_heads, p->head_dim = head_dim;
    const int32_t group_rows = n_q_heads / n_heads, part_rows = group_rows < 16 ? group_rows : 16;
    const size_t row = part_row(head_dim), blocks = (size_t)sm_count() * 2, warps = blocks * ATTEND_WARPS;
    const size_t rows = (size_t)(max_tokens < MAX_TOKENS ? max_tokens : MAX_TOKENS) * n_q_heads * row;
    // (pairs of a launch: a token's blocks of rows have 8 rows at least, a group's shared ones 16)
    const size_t pairs = (size_t)MAX_TOKENS * n_heads * ((group_rows + 7) / 8);
    int32_t rc = dev_alloc(&p->shared, (size_t)MAX_TOKENS);
    if (rc == WG_OK) rc = dev_alloc(&p->shared_cuts, pairs);
    if (rc == WG_OK) rc = dev_alloc(&p->own_cuts, pairs);
    if (rc == WG_OK) rc = dev_alloc(&p->block_parts, blocks * 2 * PART_ROWS * row);
    if (rc == WG_OK) rc = dev_alloc(&p->warp_parts, warps * 2 * part_rows * row);
    if (rc == WG_OK) rc = dev_alloc(&p->shared_rows, rows);
    if (rc == WG_OK) rc = dev_alloc(&p->own_rows, rows);
    if (rc != WG_OK) {
        wg_attend_free(p);
        return rc;
    }
    *out = p;
    return WG_OK;
}

void wg_attend_free(wg_attend *p) {
    if (!p) return;
    for (void *q : {(void *)p->shared, (void *)p->shared_cuts, (void *)p->own_cuts, (void *)p->block_parts, (void *)p->warp_parts, (void *)p->shared_rows, (void *)p->own_rows})
        cudaFree(q);
    delete p;
}

int32_t wg_kv_attend(wg_attend *attend, const wg_kv_cache *cache, const void *q, int64_t q_stride, void *out, int64_t out_stride,
                     float *lse, int32_t dtype, int32_t n_q_heads, const int32_t *table, int64_t table_stride, int32_t max_blocks,
                     const int32_t *len, int32_t n_seq, const int32_t *seq, const int32_t *pos, const int64_t *slot,
                     int32_t n_tokens, float scale, int32_t window, int32_t group, void *stream) {
    NvtxRange nvtx_range("wg_kv_attend");
    if (!attend || !cache_ok(cache) || n_tokens < 0 || n_tokens > attend->max_tokens) return WG_ERR_ARG;
    if (dtype != WG_DTYPE_BF16 && dtype != WG_DTYPE_FP16) return WG_ERR_ARG;
    if (cache->storage <= WG_KV_FP16 && (cache->storage == WG_KV_FP16) != (dtype == WG_DTYPE_FP16)) return WG_ERR_ARG;
    if (n_q_heads != attend->n_q_heads || cache->n_heads != attend->n_heads || cache->head_dim != attend->head_dim) return WG_ERR_ARG;
    if (!table || max_blocks < 1 || table_stride < max_blocks || n_seq < 1) return WG_ERR_ARG;
    const bool mapped = seq != nullptr;
    if (mapped != (pos != nullptr) || mapped != (slot != nullptr) || (!mapped && (!len || n_tokens > n_seq))) return WG_ERR_ARG;
    if (window < 0 || group < 1 || group > WG_BEAM_MAX_BEAMS || !std::isfinite(scale * LOG2_E)) return WG_ERR_ARG;
    if (n_tokens == 0) return WG_OK;
    const int64_t width = (int64_t)n_q_heads * cache->head_dim;
    if (!rows_ok(q, q_stride, width) || !rows_ok(out, out_stride, width)) return WG_ERR_ARG;
    const CacheDev c = cache_dev(cache);
    const int32_t rows = n_q_heads / cache->n_heads, row_blocks = rows <= 8 ? 1 : (rows + 15) / 16;
    const int64_t room = (int64_t)max_blocks * cache->block_size, most_tokens = room < (1ll << 31) ? room : 1ll << 31;
    const int64_t tiles = (most_tokens + 15) / 16 * row_blocks * cache->n_heads;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    const int32_t most = MAX_TOKENS / group * group;       // tokens of a launch
    for (int64_t t0 = 0; t0 < n_tokens; t0 += most) {
        AttendArgs a{};
        a.n_tokens = (int32_t)(n_tokens - t0 < most ? n_tokens - t0 : most);
        a.q = static_cast<const uint16_t *>(q) + t0 * q_stride, a.q_stride = q_stride;
        a.out = static_cast<uint16_t *>(out) + t0 * out_stride, a.out_stride = out_stride;
        a.lse = lse ? lse + t0 * n_q_heads : nullptr;
        a.table = table, a.stride = table_stride, a.max_blocks = max_blocks, a.n_seq = n_seq;
        if (mapped) {
            a.seq = seq + t0, a.pos = pos + t0, a.slot = slot + t0;
        } else {
            a.table += t0 * table_stride, a.len = len + t0, a.n_seq -= (int32_t)t0;
        }
        a.window = window, a.n_q_heads = n_q_heads, a.rows = rows, a.row_blocks = row_blocks;
        a.group = group, a.n_groups = (a.n_tokens + group - 1) / group;
        a.q_bf16 = dtype == WG_DTYPE_BF16;
        a.scale = scale * LOG2_E;
        a.together = cache->n_heads % 4 == 0 ? 4 : cache->n_heads % 2 == 0 ? 2 : 1;
        a.part_rows = rows < 16 ? rows : 16;
        a.shared = attend->shared, a.shared_cuts = attend->shared_cuts, a.own_cuts = attend->own_cuts;
        a.block_parts = attend->block_parts, a.warp_parts = attend->warp_parts, a.shared_rows = attend->shared_rows, a.own_rows = attend->own_rows;
        const int64_t most_tiles = tiles * a.n_tokens;
        int32_t rc;
        switch (cache->storage) {
            case WG_KV_BF16: rc = attend_bf16(c, a, most_tiles, st); break;
            case WG_KV_FP16: rc = attend_fp16(c, a, most_tiles, st); break;
            case WG_KV_E4M3: rc = attend_e4m3(c, a, most_tiles, st); break;
            default: rc = attend_int8(c, a, most_tiles, st); break;
        }
        if (rc != WG_OK) return rc;
    }
    return WG_OK;
}

}  // extern "C"
