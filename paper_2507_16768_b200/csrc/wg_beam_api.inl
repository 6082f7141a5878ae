// Host side of constrained beam search (wg_beam_* of wg.h).  Part of wg_api.cu's translation unit:
// the step launches that file's lookup and build kernels on the context.

struct wg_beam {
    int32_t V = 0, max_requests = 0, max_beams = 0, max_out = 0;
    int32_t chunk_stride = 0;
    float *chunk_max = nullptr;
    float2 *parts = nullptr;
    int32_t *next_item = nullptr;
};

namespace {

constexpr size_t SCAN_COUNTERS = SCAN_GROUPS * SCAN_COUNTER * sizeof(int32_t);

// Spans of 2048 positions per row, for the worst alignment of a row (it may begin up to 7 elements into
// a piece).
int32_t beam_spans(int32_t V) { return (V + 7 + 2047) / 2048; }

template <typename E, int NORM, bool CTX>
cudaError_t launch_beam_scan(const BeamArgs &a, const CtxDev &ctx, unsigned grid, cudaStream_t st) {
    return launch_pdl(beam_scan_kernel<E, NORM, CTX>, dim3(grid), dim3(BEAM_THREADS), st, a, ctx);
}

template <typename E, int NORM, bool CTX>
cudaError_t launch_beam_small(const BeamArgs &a, const CtxDev &ctx, const VocabDev &v, const BeamStepArgs &step,
                              int32_t n_req, unsigned cluster, float *score_out, int32_t *parent_out, int32_t *token_out,
                              cudaStream_t st) {
    if (cluster > 8) {                     // beyond what every device grants
        static std::atomic<uint64_t> done{0};
        const cudaError_t e = set_once(done, beam_small_kernel<E, NORM, CTX>, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
        if (e != cudaSuccess) return e;
    }
    return launch_cluster(beam_small_kernel<E, NORM, CTX>, cluster, (unsigned)n_req, PICK_THREADS, 0, st, a, ctx, v,
                          step, score_out, parent_out, token_out);
}

template <typename E, bool CTX>
int32_t launch_scan_and_pick(const BeamArgs &a, const CtxDev &ctx, const VocabDev &v, const BeamStepArgs &step,
                             int32_t n_req, unsigned grid, float *score_out, int32_t *parent_out, int32_t *token_out,
                             cudaStream_t st) {
    if (a.norm == WG_BEAM_NORM_ALLOWED)
        WG_CUDA((launch_beam_scan<E, WG_BEAM_NORM_ALLOWED, CTX>(a, ctx, grid, st)));
    else if (a.norm == WG_BEAM_NORM_FULL)
        WG_CUDA((launch_beam_scan<E, WG_BEAM_NORM_FULL, CTX>(a, ctx, grid, st)));
    else
        WG_CUDA((launch_beam_scan<E, WG_BEAM_NORM_NONE, CTX>(a, ctx, grid, st)));
    WG_LAUNCHED();
    WG_CUDA(launch_pdl(beam_pick_kernel<E, CTX>, dim3((unsigned)n_req), dim3(PICK_THREADS), st, a, ctx, v,
                       step, score_out, parent_out, token_out));
    WG_LAUNCHED();
    return WG_OK;
}

template <typename E, bool CTX>
int32_t launch_beam(const BeamArgs &a, const CtxDev &ctx, const VocabDev &v, const BeamStepArgs &step,
                    int32_t n_req, unsigned grid, float *score_out, int32_t *parent_out, int32_t *token_out,
                    cudaStream_t st) {
    // One launch where a cluster has a warp for every step of a request and the clusters find room at once:
    // 6.8 us instead of 9.4 for a call on 1 x 4 beams x 32000 (2.5 us are the host's second launch; recorded,
    // both take 6.6), 8.2 instead of 9.5 on 1 x 16.  Clusters of 16 need that many places
    // side by side and start later: with 8 requests 9.0 us instead of 8.4 recorded, so they are for few.
    unsigned cluster = 1;
    while (cluster <= SMALL_CLUSTER && cluster * PICK_WARPS < a.n_beam * a.per_row.d) cluster *= 2;
    if (cluster <= SMALL_CLUSTER && (long long)n_req * cluster <= (cluster > 8 ? sm_count() / 2 : sm_count())) {
        if (a.norm == WG_BEAM_NORM_ALLOWED)
            WG_CUDA((launch_beam_small<E, WG_BEAM_NORM_ALLOWED, CTX>(a, ctx, v, step, n_req, cluster, score_out, parent_out, token_out, st)));
        else if (a.norm == WG_BEAM_NORM_FULL)
            WG_CUDA((launch_beam_small<E, WG_BEAM_NORM_FULL, CTX>(a, ctx, v, step, n_req, cluster, score_out, parent_out, token_out, st)));
        else
            WG_CUDA((launch_beam_small<E, WG_BEAM_NORM_NONE, CTX>(a, ctx, v, step, n_req, cluster, score_out, parent_out, token_out, st)));
        WG_LAUNCHED();
        return WG_OK;
    }
    const int32_t rc = launch_scan_and_pick<E, CTX>(a, ctx, v, step, n_req, grid, score_out, parent_out, token_out, st);
    // the pick sets the counters back that the scan takes its items from: where it was not launched, this does
    if (rc != WG_OK) cudaMemsetAsync(a.next_item, 0, SCAN_COUNTERS, st);
    return rc;
}

// The scan's grid (as many blocks as are resident at once, or a step per warp) and the items it deals out:
// the last one and a half steps of every warp one by one, the step before those in twos.
unsigned beam_grid(BeamArgs &a, int32_t rows, int32_t dtype) {
    const int step = dtype == WG_DTYPE_BF16 ? ScanShape<uint16_t>::STEP : ScanShape<uint32_t>::STEP;
    a.per_row = Divisor::of((uint32_t)(((long long)a.V + 7 + step - 1) / step));
    a.n_steps = (uint32_t)rows * a.per_row.d;
    const uint32_t blocks = std::min((a.n_steps + BEAM_WARPS - 1) / BEAM_WARPS, (uint32_t)sm_count() * BEAM_BLOCKS);
    const uint32_t warps = blocks * BEAM_WARPS;
    const uint32_t ones = std::min(a.n_steps, warps * 3 / 2), twos = std::min(a.n_steps - ones, warps);
    a.n_two = twos / 2;
    a.n_long = (a.n_steps - ones - twos) / SCAN_LONG;
    a.more = a.n_steps - (SCAN_LONG - 1) * a.n_long - a.n_two > warps;
    a.groups = a.more ? SCAN_GROUPS : 1;   // (more items than warps: the whole grid, which the groups divide)
    a.per_group = blocks / a.groups;
    a.chunk_log2 = 5;
    while (a.chunk_log2 < 9 && (1 << a.chunk_log2) < a.chunk_stride) ++a.chunk_log2;
    return blocks;
}

bool beam_sizes_ok(const wg_beam *beam, int32_t n_req, int32_t n_beam, int32_t n_out, int32_t norm) {
    return beam && n_req >= 1 && n_req <= beam->max_requests && n_beam >= 1 && n_beam <= beam->max_beams &&
           n_out >= 1 && n_out <= beam->max_out && norm >= WG_BEAM_NORM_ALLOWED && norm <= WG_BEAM_NORM_NONE;
}

bool elem_aligned(const void *p, int32_t dtype) {
    return (uintptr_t)p % (dtype == WG_DTYPE_BF16 ? 2 : 4) == 0;
}

}  // namespace

extern "C" {

int32_t wg_beam_create(int32_t V, int32_t max_requests, int32_t max_beams, int32_t max_out, wg_beam **out) {
    NvtxRange nvtx_range("wg_beam_create");
    if (!out) return WG_ERR_ARG;
    *out = nullptr;
    if (V < 1 || V > INT32_MAX - 4096 || max_requests < 1 || max_beams < 1 || max_beams > WG_BEAM_MAX_BEAMS ||
        max_out < 1 || max_out > WG_BEAM_MAX_OUT || (int64_t)max_requests * max_beams > WG_MAX_ROWS ||
        (int64_t)V * max_beams >= (1LL << 32) ||
        (int64_t)max_requests * max_beams * beam_spans(V) * 2 >= (1LL << 31))   // items have 32-bit numbers
        return WG_ERR_ARG;
    wg_beam *b = new (std::nothrow) wg_beam();
    if (!b) return WG_ERR_ARG;
    b->V = V;
    b->max_requests = max_requests;
    b->max_beams = max_beams;
    b->max_out = max_out;
    b->chunk_stride = beam_spans(V) * 4;
    const size_t rows = (size_t)max_requests * max_beams;
    int32_t rc = dev_alloc(&b->chunk_max, rows * b->chunk_stride);
    if (rc == WG_OK) rc = dev_alloc(&b->parts, rows * beam_spans(V) * 2);   // (an fp32 span is two steps)
    if (rc == WG_OK) rc = dev_alloc(&b->next_item, SCAN_GROUPS * SCAN_COUNTER);
    // (the first call may be on a stream that does not wait for the default one)
    if (rc == WG_OK && (cudaMemset(b->next_item, 0, SCAN_COUNTERS) != cudaSuccess || cudaStreamSynchronize(cudaStreamLegacy) != cudaSuccess))
        rc = WG_ERR_CUDA;
    if (rc != WG_OK) {
        wg_beam_free(b);
        return rc;
    }
    *out = b;
    return WG_OK;
}

void wg_beam_free(wg_beam *b) {
    if (!b) return;
    cudaFree(b->chunk_max);   // (waits for queued work)
    cudaFree(b->parts);
    cudaFree(b->next_item);
    delete b;
}

int32_t wg_beam_select(wg_beam *beam, const void *logits, int32_t dtype, int64_t row_stride_elems,
                       const uint32_t *bitmask, int64_t mask_stride_words, const float *score,
                       const int32_t *finished, int32_t eos_id, int32_t n_req, int32_t n_beam,
                       int32_t n_out, int32_t norm, float *score_out, int32_t *parent_out,
                       int32_t *token_out, void *stream) {
    NvtxRange nvtx_range("wg_beam_select");
    if (!beam_sizes_ok(beam, n_req, n_beam, n_out, norm) || !logits || !score || !score_out || !parent_out ||
        !token_out)
        return WG_ERR_ARG;
    if (dtype != WG_DTYPE_BF16 && dtype != WG_DTYPE_FP32) return WG_ERR_ARG;
    const int32_t V = beam->V, W = (V + 31) / 32;
    if (row_stride_elems < V || !elem_aligned(logits, dtype) || (bitmask && mask_stride_words < W))
        return WG_ERR_ARG;
    if (finished && (eos_id < 0 || eos_id >= V)) return WG_ERR_ARG;
    if (score_out == score && n_out != n_beam) return WG_ERR_ARG;
    BeamArgs a{logits, row_stride_elems, bitmask, mask_stride_words, score, finished, nullptr, nullptr,
               n_beam, V, W, n_out, eos_id, norm, 0u, 0u, 0u, 0u, 0u, false, Divisor{}, beam->chunk_stride, 0, beam->chunk_max, beam->parts,
               beam->next_item};
    const unsigned grid = beam_grid(a, n_req * n_beam, dtype);
    const CtxDev none{};
    const VocabDev no_vocab{};
    const BeamStepArgs no_step{};
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    return dtype == WG_DTYPE_BF16
        ? launch_beam<uint16_t, false>(a, none, no_vocab, no_step, n_req, grid, score_out, parent_out, token_out, st)
        : launch_beam<uint32_t, false>(a, none, no_vocab, no_step, n_req, grid, score_out, parent_out, token_out, st);
}

int32_t wg_beam_step(wg_beam *beam, wg_ctx *c, int32_t *gid, int32_t *sid, float *score, int32_t n_req,
                     int32_t n_beam, const void *logits, int32_t dtype, int64_t row_stride_elems,
                     uint32_t *bitmask, int64_t mask_stride_words, int32_t norm, int32_t *parent_out,
                     int32_t *token_out, int32_t *status, uint32_t flags, void *stream) {
    NvtxRange nvtx_range("wg_beam_step");
    if (!beam_sizes_ok(beam, n_req, n_beam, n_beam, norm) || !c || !gid || !sid || !score || !logits ||
        !bitmask || !parent_out || !token_out)
        return WG_ERR_ARG;
    if (dtype != WG_DTYPE_BF16 && dtype != WG_DTYPE_FP32) return WG_ERR_ARG;
    if (flags & ~(uint32_t)WG_NO_CACHE) return WG_ERR_ARG;
    const VocabDev &v = c->vocab->dev;
    const int32_t rows = n_req * n_beam;
    if (beam->V != v.V || !batch_ok(c, rows)) return WG_ERR_ARG;
    if (row_stride_elems < v.V || !elem_aligned(logits, dtype) || mask_stride_words < v.W) return WG_ERR_ARG;
    const bool no_cache = (flags & WG_NO_CACHE) != 0;
    if (!no_cache && c->part_end != 0) return WG_ERR_ARG;  // cached masks are partial: see wg_decode_step_shard
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    // the rows' masks, as the first launches of a decode step
    BuildWork work{};
    if (no_cache) {
        WG_CUDA(launch_pdl(reset_rows_kernel, dim3((rows + 255) / 256), dim3(256), st, c->dev, rows));
        work = BuildWork{gid, sid, nullptr, bitmask, mask_stride_words, nullptr, rows, 0, 0, 0};
    } else {
        WG_CUDA(launch_pdl(cache_lookup_insert_kernel, dim3(1), dim3(1024), st, c->dev, gid, sid, rows,
                           bitmask, mask_stride_words));
        work = BuildWork{c->dev.bl_gid, c->dev.bl_sid, c->dev.bl_dst, nullptr, 0, c->dev.bl_count, 0, 0, 0, 0};
    }
    WG_LAUNCHED();
    const int32_t rc = launch_build(c, work, rows, st, true);
    if (rc != WG_OK) return rc;
    BeamArgs a{logits, row_stride_elems, bitmask, mask_stride_words, score, nullptr, gid, sid,
               n_beam, v.V, v.W, n_beam, v.eos_id, norm, 0u, 0u, 0u, 0u, 0u, false, Divisor{}, beam->chunk_stride, 0, beam->chunk_max, beam->parts,
               beam->next_item};
    const unsigned grid = beam_grid(a, rows, dtype);
    const BeamStepArgs step{gid, sid, status};
    return dtype == WG_DTYPE_BF16
        ? launch_beam<uint16_t, true>(a, c->dev, v, step, n_req, grid, score, parent_out, token_out, st)
        : launch_beam<uint32_t, true>(a, c->dev, v, step, n_req, grid, score, parent_out, token_out, st);
}

int32_t wg_beam_backtrack(const int32_t *token, const int32_t *parent, int32_t n_steps, int32_t n_req,
                          int32_t n_beam, int32_t *out, void *stream) {
    NvtxRange nvtx_range("wg_beam_backtrack");
    if (n_steps < 0 || n_req < 1 || n_req > WG_MAX_ROWS || n_beam < 1 || n_beam > WG_BEAM_MAX_BEAMS)
        return WG_ERR_ARG;
    if (n_steps == 0) return WG_OK;
    if (!token || !parent || !out) return WG_ERR_ARG;
    BackArgs a{token, parent, out, n_steps, n_req, n_beam, 32 / n_beam, 0};
    int parts = 1;
    while (parts < BACK_CLUSTER && parts * BACK_STEPS < n_steps) parts <<= 1;
    a.steps = std::min(BACK_STEPS, (n_steps + parts - 1) / parts);
    static std::atomic<uint64_t> done{0};
    WG_CUDA(set_once(done, beam_backtrack_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)sizeof(BackShared)));
    WG_CUDA(launch_cluster(beam_backtrack_kernel, (unsigned)parts, (unsigned)((n_req + a.group - 1) / a.group), BACK_THREADS,
                           sizeof(BackShared), static_cast<cudaStream_t>(stream), a));
    WG_LAUNCHED();
    return WG_OK;
}

}  // extern "C"
