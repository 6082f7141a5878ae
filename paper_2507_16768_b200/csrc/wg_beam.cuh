// Device code of constrained beam search: the scan of the logits, the selection, the way back.
//
// Mathematics.  Row i = (request r, beam b) has logits x, allowed tokens A and a running score c.
// With m = max of x over the tokens in the denominator and s = sum of exp(x - m), lse = m + log s,
// and a candidate's score is c + (x[t] - lse).  The n_out best of a request are found without ever
// writing scores out:
//   * the scan reads every logit once and keeps, per chunk of 256 tokens, the largest allowed logit,
//     and per warp (m, s) with the running-maximum rescaling of an online softmax;
//   * a score is a non-decreasing function of the logit within a row (two fp32 roundings, both
//     monotonic), so a chunk's best score is the score of its largest logit.  Rank the chunks of all
//     beams by (best score, then the lower chunk number).  An element outside the first n_out
//     chunks is beaten by the best element of each of them: by score, or at equal scores by index,
//     since a chunk before it holds lower indices only.  So the n_out best elements lie in the first
//     n_out chunks, and those 256 * n_out elements are all that the pick reads again.
#pragma once

#include "wg_kernels.cuh"

constexpr int BEAM_THREADS = 256;           // scan
constexpr int BEAM_WARPS = BEAM_THREADS / 32;
constexpr int BEAM_SPANS_PER_WARP = 4;      // a block covers at most 8 * 4 spans of 1024 tokens
constexpr int BEAM_CHUNK = 256;             // tokens per chunk maximum
constexpr int PICK_THREADS = 512;
constexpr int PICK_GROUPS = 128;            // four threads each
constexpr int PICK_LIST = 512;              // candidates that are ranked against each other

struct BeamArgs {
    const void *logits;
    int64_t row_stride;       // elements
    const uint32_t *bitmask;  // NULL: everything is allowed (never with a context)
    int64_t mask_stride;      // words
    const float *score;
    const int32_t *finished;  // or NULL
    const int32_t *gid, *sid; // with a context: the rows' states (finished = DONE)
    int32_t n_beam, V, W, n_out, eos, norm;
    int32_t spans_per_block;
    int32_t n_parts;          // (max, sum) pairs per row: scan blocks per row * BEAM_WARPS
    int32_t chunk_stride;     // chunk maxima per row (four per span)
    float *chunk_max;         // [rows][chunk_stride]
    float2 *parts;            // [rows][n_parts]
};

// What a step under grammars does with the selection.
struct BeamStepArgs {
    int32_t *gid, *sid;
    int32_t *status;          // or NULL
};

enum { BEAM_ROW_DEAD = 0, BEAM_ROW_LIVE = 1, BEAM_ROW_FINISHED = 2 };

// What a row can offer: nothing (no hypothesis), one candidate (finished), or its tokens.
template <bool CTX>
__device__ __forceinline__ int beam_row_kind(const BeamArgs &a, const CtxDev &ctx, int row, float score) {
    if (!(score > -INFINITY)) return BEAM_ROW_DEAD;     // (NaN too)
    if (CTX) {
        const int g = a.gid[row], s = a.sid[row];
        if (g >= 0 && g < ctx.n_grammars && s > 0 && s == ctx.grammars[g].done) return BEAM_ROW_FINISHED;
        return BEAM_ROW_LIVE;
    }
    return a.finished && a.finished[row] ? BEAM_ROW_FINISHED : BEAM_ROW_LIVE;
}

// Where a row's packed mask is: a row of words, a compact cache entry, or nowhere (all allowed).
struct MaskSource {
    const uint32_t *words;
    const uint2 *hdr;
    const uint32_t *arena;
    int V, W;

    // Word w, zero outside the row; bits at and beyond V are 0.
    __device__ __forceinline__ uint32_t word(int w) const {
        if (w < 0 || w >= W) return 0u;
        if (hdr) return entry_word(hdr, arena, w >> 5, w & 31, V, W);
        const uint32_t full = full_word(w, V, W);
        return words ? words[w] & full : full;
    }
};

template <bool CTX>
__device__ __forceinline__ MaskSource mask_source(const BeamArgs &a, const CtxDev &ctx, int row) {
    MaskSource m{a.bitmask ? a.bitmask + (int64_t)row * a.mask_stride : nullptr, nullptr, nullptr, a.V, a.W};
    if (CTX) {
        const int32_t slot = ctx.slot[row];
        if (slot >= 0 && !ctx.compact) {
            m.words = ctx.pool + (int64_t)slot * ctx.pool_stride;
        } else if (slot >= 0 && ctx.ent_fail[slot]) {   // built in this call, no room in the arena
            m.words = ctx.stage + (int64_t)ctx.ent_stage[slot] * ctx.pool_stride;
        } else if (slot >= 0) {
            m.hdr = ctx.ent_hdr + (int64_t)slot * ctx.hdr_stride;
            m.arena = ctx.arena;
        }
    }
    return m;
}

// A row seen as 16-byte pieces: `base` is the row's address rounded down to 16 bytes, `off` how many
// elements that is.  Position p of the view is token p - off, so every piece is one aligned load
// whatever the row's alignment; spans and chunks are counted in positions.
template <typename E>
struct RowView {
    const E *base;
    int off, V;

    __device__ __forceinline__ RowView(const void *logits, int64_t stride, int row, int V_) : V(V_) {
        const E *p = static_cast<const E *>(logits) + (int64_t)row * stride;
        off = (int)(((uintptr_t)p & 15) / sizeof(E));
        base = p - off;
    }

    // The 16 bytes at position p (a multiple of the piece size); elements outside the row are -inf.
    __device__ __forceinline__ uint4 piece(int p) const {
        constexpr int EPC = ElemTraits<E>::PER_CHUNK;
        if (p >= off && p + EPC <= V + off) {
            uint4 v;
            asm volatile("ld.global.L1::no_allocate.v4.u32 {%0, %1, %2, %3}, [%4];"
                         : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(base + p));
            return v;
        }
        // the row's ragged ends: element by element, nothing outside the row is touched
        uint32_t w[4] = {0, 0, 0, 0};
#pragma unroll 1
        for (int i = EPC - 1; i >= 0; --i) {
            const uint32_t e = (p + i >= off && p + i < V + off) ? (uint32_t)base[p + i]
                                                                : (uint32_t)ElemTraits<E>::NEG_INF;
            if (sizeof(E) == 2) {
                w[3] = __funnelshift_l(w[2], w[3], 16);
                w[2] = __funnelshift_l(w[1], w[2], 16);
                w[1] = __funnelshift_l(w[0], w[1], 16);
                w[0] = (w[0] << 16) | e;
            } else {
                w[3] = w[2]; w[2] = w[1]; w[1] = w[0]; w[0] = e;
            }
        }
        return make_uint4(w[0], w[1], w[2], w[3]);
    }
};

// Mask bits of the 32 positions from position 32 * w on.
__device__ __forceinline__ uint32_t shifted_word(const MaskSource &m, int w, int off) {
    if (off == 0) return m.word(w);
    return __funnelshift_l(m.word(w - 1), m.word(w), off);
}

// Disallowed elements of a piece become -inf.  bit i of `bits` belongs to element i.
template <typename E>
__device__ __forceinline__ void mask_piece(uint32_t (&w)[4], uint32_t bits) {
    if (sizeof(E) == 2) {
        // bit i of a group of four to the top of byte i (the partial products do not overlap), then
        // a byte permute that spreads that top bit over the element's two bytes
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const uint32_t t = ((bits >> (4 * h)) & 0xFu) * 0x10204080u;
            uint32_t lo, hi;    // (the intrinsic knows no sign spreading)
            asm("prmt.b32 %0, %1, 0, 0x9988;" : "=r"(lo) : "r"(t));
            asm("prmt.b32 %0, %1, 0, 0xBBAA;" : "=r"(hi) : "r"(t));
            w[2 * h] = (w[2 * h] & lo) | (NEG_INF_BF16X2 & ~lo);
            w[2 * h + 1] = (w[2 * h + 1] & hi) | (NEG_INF_BF16X2 & ~hi);
        }
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = ((bits >> i) & 1u) ? w[i] : NEG_INF_F32;
    }
}

// Largest element of a piece (NaN elements are passed over unless there is nothing else).
template <typename E>
__device__ __forceinline__ float piece_max(const uint32_t (&w)[4]) {
    if (sizeof(E) == 2) {
        const uint32_t u = bf162_bits(__hmax2(__hmax2(as_bf162(w[0]), as_bf162(w[1])),
                                              __hmax2(as_bf162(w[2]), as_bf162(w[3]))));
        return fmaxf(__uint_as_float(u << 16), __uint_as_float(u & 0xFFFF0000u));
    }
    return fmaxf(fmaxf(__uint_as_float(w[0]), __uint_as_float(w[1])),
                 fmaxf(__uint_as_float(w[2]), __uint_as_float(w[3])));
}

__device__ __forceinline__ float warp_max(float x) {
    float r;
    asm volatile("redux.sync.max.f32 %0, %1, 0xffffffff;" : "=f"(r) : "f"(x));
    return r;
}

// 2^x with the special-function unit: about 2 ulp; the 20 or so bits that are left of a term are
// far more than its weight in a sum of thousands needs, and the sum itself is kept in fp32.
__device__ __forceinline__ float exp2_fast(float x) {
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}

constexpr float LOG2_E = 1.4426950408889634f;

// Sum of exp(x - m) over a piece.  The difference is formed before it is scaled: a row whose
// largest logit is the type's lowest value must still give exp(0) for it.
template <typename E>
__device__ __forceinline__ void piece_exp(const uint32_t (&w)[4], float m, float &s0, float &s1) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if (sizeof(E) == 2) {
            s0 += exp2_fast((__uint_as_float(w[i] << 16) - m) * LOG2_E);
            s1 += exp2_fast((__uint_as_float(w[i] & 0xFFFF0000u) - m) * LOG2_E);
        } else if (i & 1) {
            s1 += exp2_fast((__uint_as_float(w[i]) - m) * LOG2_E);
        } else {
            s0 += exp2_fast((__uint_as_float(w[i]) - m) * LOG2_E);
        }
    }
}

// ---------------------------------------------------------------------------------------
// Scan.  grid = (blocks per row, rows); a warp takes spans of 1024 positions, 2 KB (four 16-byte
// loads per lane) at a time, the next 2 KB requested before the current are worked on.
// ---------------------------------------------------------------------------------------
template <typename E, int NORM, bool CTX>
__global__ void __launch_bounds__(BEAM_THREADS)
beam_scan_kernel(BeamArgs a, CtxDev ctx) {
    constexpr int EPC = ElemTraits<E>::PER_CHUNK;
    constexpr int GROUP = 4;                                  // loads per lane and step
    constexpr int STEPS = 1024 / (32 * EPC * GROUP);          // steps per span: 1 (bf16), 2 (fp32)
    constexpr int PER_CHUNK = BEAM_CHUNK / (32 * EPC);        // loads per chunk: 1, 2
    constexpr int CHUNKS = GROUP / PER_CHUNK;                 // chunks per step: 4, 2
    constexpr uint32_t ALL = (1u << EPC) - 1u;
    pdl_enter();
    const int row = blockIdx.y;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    if (beam_row_kind<CTX>(a, ctx, row, a.score[row]) != BEAM_ROW_LIVE) return;
    const RowView<E> x(a.logits, a.row_stride, row, a.V);
    const MaskSource mask = mask_source<CTX>(a, ctx, row);
    const int n_spans = (a.V + x.off + 1023) / 1024;
    const int first = blockIdx.x * a.spans_per_block + warp;
    const int end = min((int)(blockIdx.x + 1) * a.spans_per_block, n_spans);
    uint32_t words[BEAM_SPANS_PER_WARP];
#pragma unroll
    for (int k = 0; k < BEAM_SPANS_PER_WARP; ++k) {
        const int span = first + k * BEAM_WARPS;
        words[k] = span < end ? shifted_word(mask, span * 32 + lane, x.off) : 0u;
    }
    float *chunk_row = a.chunk_max + (int64_t)row * a.chunk_stride;
    float m = -INFINITY, s0 = 0.f, s1 = 0.f;   // m is the same in all lanes

    uint4 next[GROUP];
    // requests the loads of step q of the span in slot k
    auto request = [&](int k, int q) {
        const int span = first + k * BEAM_WARPS;
#pragma unroll
        for (int i = 0; i < GROUP; ++i) {
            const int c = (q * GROUP + i) * 32 + lane;        // piece within the span
            const uint32_t word = __shfl_sync(0xFFFFFFFFu, words[k], c * EPC / 32);
            const uint32_t bits = (word >> (c * EPC % 32)) & ALL;
            next[i] = make_uint4(0, 0, 0, 0);
            if (span < end && (NORM == WG_BEAM_NORM_FULL || bits != 0u))
                next[i] = x.piece(span * 1024 + c * EPC);
        }
    };
    request(0, 0);
#pragma unroll
    for (int k = 0; k < BEAM_SPANS_PER_WARP; ++k) {
        const int span = first + k * BEAM_WARPS;
#pragma unroll
        for (int q = 0; q < STEPS; ++q) {
            uint4 v[GROUP];
#pragma unroll
            for (int i = 0; i < GROUP; ++i) v[i] = next[i];
            if (q + 1 < STEPS) request(k, q + 1);
            else if (k + 1 < BEAM_SPANS_PER_WARP) request(k + 1, 0);
            if (span >= end) continue;
            const bool some = __ballot_sync(0xFFFFFFFFu, words[k] != 0u) != 0u;
            float best[CHUNKS];
#pragma unroll
            for (int i = 0; i < CHUNKS; ++i) best[i] = -INFINITY;
            if (NORM == WG_BEAM_NORM_FULL || some) {
                uint32_t w[GROUP][4];
                float top = -INFINITY;
#pragma unroll
                for (int i = 0; i < GROUP; ++i) {
                    const int c = (q * GROUP + i) * 32 + lane;
                    const uint32_t word = __shfl_sync(0xFFFFFFFFu, words[k], c * EPC / 32);
                    const uint32_t bits = (word >> (c * EPC % 32)) & ALL;
                    uint32_t y[4] = {v[i].x, v[i].y, v[i].z, v[i].w};
                    if (NORM == WG_BEAM_NORM_FULL) {
#pragma unroll
                        for (int j = 0; j < 4; ++j) w[i][j] = y[j];
                        top = fmaxf(top, piece_max<E>(y));
                        mask_piece<E>(y, bits);
                    } else {
                        mask_piece<E>(y, bits);
#pragma unroll
                        for (int j = 0; j < 4; ++j) w[i][j] = y[j];
                    }
                    best[i / PER_CHUNK] = fmaxf(best[i / PER_CHUNK], piece_max<E>(y));
                }
#pragma unroll
                for (int i = 0; i < CHUNKS; ++i) best[i] = warp_max(best[i]);
                if (NORM != WG_BEAM_NORM_NONE) {
                    float high = m;
                    if (NORM == WG_BEAM_NORM_FULL) {
                        high = fmaxf(high, warp_max(top));
                    } else {
#pragma unroll
                        for (int i = 0; i < CHUNKS; ++i) high = fmaxf(high, best[i]);
                    }
                    if (high > m) {                            // uniform
                        const float scale = exp2_fast((m - high) * LOG2_E);
                        s0 *= scale;
                        s1 *= scale;
                        m = high;
                    }
                    if (m > -INFINITY) {
#pragma unroll
                        for (int i = 0; i < GROUP; ++i) piece_exp<E>(w[i], m, s0, s1);
                    }
                }
            }
            if (lane == 0) {
                float *dst = chunk_row + span * 4 + q * CHUNKS;
                if (CHUNKS == 4) *reinterpret_cast<float4 *>(dst) = make_float4(best[0], best[1], best[2 % CHUNKS], best[3 % CHUNKS]);
                else *reinterpret_cast<float2 *>(dst) = make_float2(best[0], best[1]);
            }
        }
    }
    if (NORM != WG_BEAM_NORM_NONE) {
        float s = s0 + s1;
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xFFFFFFFFu, s, o);
        if (lane == 0) a.parts[(int64_t)row * a.n_parts + blockIdx.x * BEAM_WARPS + warp] = make_float2(m, s);
    }
}

// ---------------------------------------------------------------------------------------
// Pick.  One block per request.
// ---------------------------------------------------------------------------------------
__device__ __forceinline__ uint32_t score_key(float s) {   // 0: not a candidate
    return s > -INFINITY ? order_key(__float_as_uint(s)) : 0u;
}

__device__ __forceinline__ float key_score(uint32_t k) {
    return __uint_as_float((k & 0x80000000u) ? (k & 0x7FFFFFFFu) : ~k);
}

__device__ __forceinline__ unsigned long long pack_key(uint32_t key, uint32_t idx) {
    return ((unsigned long long)key << 32) | (0xFFFFFFFFu - idx);
}

struct PickShared {
    unsigned long long list[PICK_LIST];
    uint32_t group[PICK_GROUPS];
    uint32_t chunk[WG_BEAM_MAX_OUT];       // the chosen chunks, best first
    int32_t parent[WG_BEAM_MAX_OUT], token[WG_BEAM_MAX_OUT];
    float score[WG_BEAM_MAX_BEAMS], lse[WG_BEAM_MAX_BEAMS];
    int32_t kind[WG_BEAM_MAX_BEAMS];
    int32_t n_written[WG_BEAM_MAX_BEAMS];  // chunk maxima the scan wrote for the row
    uint32_t bound;                        // key that n_out candidates reach
    int32_t n;
    int32_t count[PICK_THREADS / 32];
};

// Sum of v over the block, in every thread.
__device__ __forceinline__ int block_sum(PickShared &sh, int v) {
    v = __reduce_add_sync(0xFFFFFFFFu, v);
    if ((threadIdx.x & 31) == 0) sh.count[threadIdx.x >> 5] = v;
    __syncthreads();
    int total = 0;
#pragma unroll
    for (int i = 0; i < PICK_THREADS / 32; ++i) total += sh.count[i];
    __syncthreads();
    return total;
}

// Puts the candidates that `each` enumerates into sh.list: all that reach `bound`, or, where
// those are more than the list holds (many equal scores), exactly the n_out largest, found by
// bisection over the packed keys.  `each(f)` calls f(packed key) for the calling thread's share; packed
// keys are unlike one another.  Returns how many are listed.
template <typename Each>
__device__ __forceinline__ int collect(PickShared &sh, uint32_t bound, int n_out, const Each &each) {
    if (threadIdx.x == 0) sh.n = 0;
    __syncthreads();
    const unsigned long long low = (unsigned long long)bound << 32;
    each([&](unsigned long long k) {
        if (k >= low) {
            const int at = atomicAdd(&sh.n, 1);
            if (at < PICK_LIST) sh.list[at] = k;
        }
    });
    __syncthreads();
    const int n = sh.n;
    if (n <= PICK_LIST) return n;
    unsigned long long cut = 0ull;         // the largest value that n_out keys reach
    for (int bit = 63; bit >= 0; --bit) {
        const unsigned long long trial = cut | (1ull << bit);
        int mine = 0;
        each([&](unsigned long long k) { mine += k >= trial; });
        if (block_sum(sh, mine) >= n_out) cut = trial;
    }
    if (threadIdx.x == 0) sh.n = 0;
    __syncthreads();
    each([&](unsigned long long k) {
        if (k >= cut) {
            const int at = atomicAdd(&sh.n, 1);
            if (at < PICK_LIST) sh.list[at] = k;
        }
    });
    __syncthreads();
    return min(sh.n, PICK_LIST);
}

// Calls f(rank, packed key) for the listed candidates of rank below n_out (0 = the largest).
template <typename F>
__device__ __forceinline__ void ranked(const PickShared &sh, int n, int n_out, const F &f) {
    for (int i = threadIdx.x; i < n; i += PICK_THREADS) {
        const unsigned long long mine = sh.list[i];
        int rank = 0;
        for (int j = 0; j < n; ++j) rank += sh.list[j] > mine;
        if (rank < n_out) f(rank, mine);
    }
}

template <typename E, bool CTX>
__device__ __forceinline__ void beam_pick(PickShared &sh, const BeamArgs &a, const CtxDev &ctx, int req) {
    constexpr int EPC = ElemTraits<E>::PER_CHUNK;
    constexpr int PER_CHUNK = BEAM_CHUNK / (32 * EPC);
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int K = a.n_beam, row0 = req * K;
    const int n_chunks = a.chunk_stride;
    // ---- the rows' log-sum-exp from the warps' pairs
    for (int b = warp; b < K; b += PICK_THREADS / 32) {
        const int row = row0 + b;
        const float score = a.score[row];
        const int kind = beam_row_kind<CTX>(a, ctx, row, score);
        float lse = 0.f;
        if (kind == BEAM_ROW_LIVE && a.norm != WG_BEAM_NORM_NONE) {
            float m = -INFINITY, s = 0.f;
            for (int i = lane; i < a.n_parts; i += 32) {
                const float2 p = a.parts[(int64_t)row * a.n_parts + i];
                const float high = fmaxf(m, p.x);
                if (high > -INFINITY)      // (a pair that saw nothing is (-inf, 0))
                    s = s * exp2_fast((m - high) * LOG2_E) + p.y * exp2_fast((p.x - high) * LOG2_E);
                m = high;
            }
            const float high = warp_max(m);
            s = high > -INFINITY ? s * exp2_fast((m - high) * LOG2_E) : 0.f;
#pragma unroll
            for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xFFFFFFFFu, s, o);
            lse = high + logf(s);
        }
        if (lane == 0) {
            sh.score[b] = score;
            sh.lse[b] = lse;
            sh.kind[b] = kind;
            const RowView<E> x(a.logits, a.row_stride, row, a.V);
            sh.n_written[b] = kind == BEAM_ROW_LIVE ? (a.V + x.off + BEAM_CHUNK - 1) / BEAM_CHUNK : 0;
        }
    }
    __syncthreads();
    // ---- the n_out best chunks
    const int n_keys = K * n_chunks;
    auto chunk_key = [&](int i) -> uint32_t {
        const int b = i / n_chunks;
        const int c = i - b * n_chunks;
        if (c >= sh.n_written[b]) return 0u;
        return score_key(sh.score[b] + (a.chunk_max[(int64_t)(row0 + b) * n_chunks + c] - sh.lse[b]));
    };
    // a lower bound for the n_out-th largest: that of the maxima of 128 groups of threads
    uint32_t top = 0;
#pragma unroll 4
    for (int i = threadIdx.x; i < n_keys; i += PICK_THREADS) top = max(top, chunk_key(i));
    top = max(top, __shfl_xor_sync(0xFFFFFFFFu, top, 1));
    top = max(top, __shfl_xor_sync(0xFFFFFFFFu, top, 2));
    if ((lane & 3) == 0) sh.group[threadIdx.x >> 2] = top;
    __syncthreads();
    if (threadIdx.x < PICK_GROUPS) {
        const uint32_t mine = sh.group[threadIdx.x];
        int rank = 0;
#pragma unroll 8
        for (int j = 0; j < PICK_GROUPS; ++j)
            rank += sh.group[j] > mine || (sh.group[j] == mine && j < (int)threadIdx.x);
        if (rank == a.n_out - 1) sh.bound = max(mine, 1u);
    }
    __syncthreads();
    const uint32_t chunk_bound = sh.bound;
    int n = collect(sh, chunk_bound, a.n_out, [&](auto f) {
#pragma unroll 4
        for (int i = threadIdx.x; i < n_keys; i += PICK_THREADS) f(pack_key(chunk_key(i), (uint32_t)i));
    });
    if (threadIdx.x == 0) sh.bound = 1u;
    __syncthreads();
    ranked(sh, n, a.n_out, [&](int rank, unsigned long long k) {
        sh.chunk[rank] = 0xFFFFFFFFu - (uint32_t)k;
        if (rank == a.n_out - 1) sh.bound = (uint32_t)(k >> 32);   // n_out elements reach this
    });
    __syncthreads();
    // ---- the n_out best elements of those chunks, and the finished rows' candidates
    const int n_sel = min(n, a.n_out);
    const uint32_t elem_bound = sh.bound;
    n = collect(sh, elem_bound, a.n_out, [&](auto f) {
        for (int i = warp; i < n_sel; i += PICK_THREADS / 32) {
            const int at = (int)sh.chunk[i];
            const int b = at / n_chunks, p0 = (at - b * n_chunks) * BEAM_CHUNK;
            const RowView<E> x(a.logits, a.row_stride, row0 + b, a.V);
            const MaskSource mask = mask_source<CTX>(a, ctx, row0 + b);
            const float score = sh.score[b], lse = sh.lse[b];
#pragma unroll
            for (int q = 0; q < PER_CHUNK; ++q) {
                const int p = p0 + (q * 32 + lane) * EPC;
                const uint32_t bits = shifted_word(mask, p >> 5, x.off) >> (p & 31);
                const uint4 v = x.piece(p);
                const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
                for (int j = 0; j < EPC; ++j) {
                    const uint32_t e = sizeof(E) == 2
                        ? ((j & 1) ? (w[j >> 1] & 0xFFFF0000u) : (w[j >> 1] << 16)) : w[j];
                    const uint32_t key = ((bits >> j) & 1u) ? score_key(score + (__uint_as_float(e) - lse)) : 0u;
                    f(pack_key(key, (uint32_t)b * (uint32_t)a.V + (uint32_t)(p + j - x.off)));
                }
            }
        }
        if ((int)threadIdx.x < K && sh.kind[threadIdx.x] == BEAM_ROW_FINISHED)
            f(pack_key(score_key(sh.score[threadIdx.x]), threadIdx.x * (uint32_t)a.V + (uint32_t)a.eos));
    });
}

template <typename E, bool CTX>
__global__ void __launch_bounds__(PICK_THREADS)
beam_pick_kernel(BeamArgs a, CtxDev ctx, VocabDev v, BeamStepArgs st, float *score_out,
                 int32_t *parent_out, int32_t *token_out) {
    __shared__ PickShared sh;
    pdl_enter();
    const int req = blockIdx.x;
    beam_pick<E, CTX>(sh, a, ctx, req);
    const int n = min(sh.n, PICK_LIST);
    // ---- out, best first
    const int64_t out0 = (int64_t)req * a.n_out;
    if ((int)threadIdx.x < a.n_out && (int)threadIdx.x >= n) {
        score_out[out0 + threadIdx.x] = -INFINITY;
        parent_out[out0 + threadIdx.x] = sh.parent[threadIdx.x] = -1;
        token_out[out0 + threadIdx.x] = sh.token[threadIdx.x] = -1;
    }
    ranked(sh, n, a.n_out, [&](int rank, unsigned long long k) {
        const uint32_t flat = 0xFFFFFFFFu - (uint32_t)k;
        const uint32_t b = flat / (uint32_t)a.V;
        score_out[out0 + rank] = key_score((uint32_t)(k >> 32));
        parent_out[out0 + rank] = sh.parent[rank] = (int32_t)b;
        token_out[out0 + rank] = sh.token[rank] = (int32_t)(flat - b * (uint32_t)a.V);
    });
    if (!CTX) return;
    // ---- the states follow: every row takes its parent's, walked over the chosen token
    __syncthreads();
    const int row0 = req * a.n_beam, j = (int)threadIdx.x;
    int32_t g = 0, next = 0;
    const bool chosen = j < a.n_beam && sh.parent[j] >= 0;
    if (chosen) {
        g = st.gid[row0 + sh.parent[j]];
        const uint32_t s = (uint32_t)st.sid[row0 + sh.parent[j]];
        const int t = sh.token[j];
        const GrammarDev gr = ctx.grammars[g];   // (a row of an unknown grammar has no candidates)
        if (gr.forced && gr.forced[s].x >= 0)
            next = gr.forced[s].y;
        else if (t == v.eos_id)
            next = gr.wide ? (int32_t)static_cast<const uint32_t *>(gr.table)[(size_t)s * gr.n_classes + gr.eos_class]
                           : (int32_t)static_cast<const uint16_t *>(gr.table)[(size_t)s * gr.n_classes + gr.eos_class];
        else
            next = gr.wide
                ? (int32_t)walk_token_classes<uint32_t>(v, gr.rec_class, static_cast<const uint32_t *>(gr.table),
                                                        gr.n_classes, gr.byte_class, s, t)
                : (int32_t)walk_token_classes<uint16_t>(v, gr.rec_class, static_cast<const uint16_t *>(gr.table),
                                                        gr.n_classes, gr.byte_class, s, t);
    }
    __syncthreads();   // everybody has read the old states
    if (j < a.n_beam) {
        if (chosen) {
            st.gid[row0 + j] = g;
            st.sid[row0 + j] = next;
        } else {
            atomicAdd(&ctx.stats[ST_EMPTY], 1ull);
        }
        if (st.status) st.status[row0 + j] = chosen ? WG_OK : WG_ERR_EMPTY_MASK;
    }
}

// ---------------------------------------------------------------------------------------
// Back-track.  One block per request walks its parents from the last step to the first.  The walk is
// a chain of dependent look-ups, so the steps are cut into segments: every segment is first walked
// from all beams at once (a map from its last beams to its first), the maps are chained, and
// then every segment is walked again from the beam that the final hypothesis really comes by.  Parents are
// staged in shared memory as bytes, a tile of steps at a time.
// ---------------------------------------------------------------------------------------
constexpr int BACK_THREADS = 512;
constexpr int BACK_DEAD = 255;

__global__ void __launch_bounds__(BACK_THREADS)
beam_backtrack_kernel(const int32_t *__restrict__ token, const int32_t *__restrict__ parent, int T,
                      int n_req, int K, int tile, int32_t *__restrict__ out) {
    extern __shared__ uint8_t back_smem[];
    uint8_t *par = back_smem;                       // [tile][K]
    uint8_t *path = par + tile * K;                 // [tile][K]: beam of step t of final beam j
    __shared__ uint8_t maps[BACK_THREADS];          // [segment][K]
    __shared__ uint8_t at[WG_BEAM_MAX_BEAMS];       // where the final beams stand before the tile
    pdl_enter();
    const int r = blockIdx.x;
    const int64_t step = (int64_t)n_req * K;        // entries per step
    const int64_t col = (int64_t)r * K;
    const int n_seg = BACK_THREADS / K;
    const int seg = (int)threadIdx.x / K, j = (int)threadIdx.x - seg * K;
    if ((int)threadIdx.x < K) at[threadIdx.x] = (uint8_t)threadIdx.x;
    for (int t1 = T; t1 > 0; t1 -= tile) {          // steps [t0, t1)
        const int t0 = max(0, t1 - tile), n = t1 - t0;
        __syncthreads();                            // the previous tile is done with
        for (int i = threadIdx.x; i < n * K; i += BACK_THREADS) {
            const int t = i / K;
            const int p = parent[(int64_t)(t0 + t) * step + col + (i - t * K)];
            par[i] = p >= 0 && p < K ? (uint8_t)p : (uint8_t)BACK_DEAD;
        }
        __syncthreads();
        const int per = (n + n_seg - 1) / n_seg;
        const int lo = min(n, seg * per), hi = min(n, lo + per);
        if (seg < n_seg) {
            int b = j;
            for (int t = hi - 1; t >= lo; --t)
                if (b != BACK_DEAD) b = par[t * K + b];
            maps[seg * K + j] = (uint8_t)b;
        }
        __syncthreads();
        if ((int)threadIdx.x < K) {                 // maps[s][j] becomes where j enters segment s
            int b = at[threadIdx.x];
            for (int s = n_seg - 1; s >= 0; --s) {
                // (a beam's own entry may be needed by its siblings: read by all, then written)
                const int to = b == BACK_DEAD ? BACK_DEAD : maps[s * K + b];
                __syncwarp((1ull << K) - 1ull);
                maps[s * K + threadIdx.x] = (uint8_t)b;
                b = to;
            }
            at[threadIdx.x] = (uint8_t)b;
        }
        __syncthreads();
        if (seg < n_seg) {
            int b = maps[seg * K + j];
            for (int t = hi - 1; t >= lo; --t) {
                path[t * K + j] = (uint8_t)b;
                if (b != BACK_DEAD) b = par[t * K + b];
            }
        }
        __syncthreads();
        for (int t = threadIdx.x; t < n; t += BACK_THREADS) {
            const int32_t *row = token + (int64_t)(t0 + t) * step + col;
            for (int jj = 0; jj < K; ++jj) {
                const int b = path[t * K + jj];
                out[(col + jj) * T + t0 + t] = b == BACK_DEAD ? -1 : row[b];
            }
        }
    }
    __syncthreads();
    for (int jj = 0; jj < K; ++jj)                  // a way back that broke off: no sequence
        if (at[jj] == BACK_DEAD)
            for (int t = threadIdx.x; t < T; t += BACK_THREADS) out[(col + jj) * T + t] = -1;
}
