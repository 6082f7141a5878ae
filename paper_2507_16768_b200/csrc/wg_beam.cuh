// Device code of constrained beam search: the scan of the logits, the selection, the way back.
//
// Mathematics.  Row i = (request r, beam b) has logits x, allowed tokens A and a running score c.
// With m = max of x over the tokens in the denominator and s = sum of exp(x - m), lse = m + log s,
// and a candidate's score is c + (x[t] - lse).  The n_out best of a request are found without ever
// writing scores out:
//   * the scan reads every logit once and keeps, per chunk of 512 tokens, the largest allowed logit,
//     and per step of a warp (4 KB of a row) its own (m, s); the pick moves the steps' sums to the row's m;
//   * a score is a non-decreasing function of the logit within a row (two fp32 roundings, both
//     monotonic), so a chunk's best score is the score of its largest logit.  Rank the chunks of all
//     beams by (best score, then the lower chunk number).  An element outside the first n_out
//     chunks is beaten by the best element of each of them: by score, or at equal scores by index,
//     since a chunk before it holds lower indices only.  So the n_out best elements lie in the first
//     n_out chunks, and those 512 * n_out elements are all that the pick reads again.
#pragma once

#include "wg_divide.cuh"
#include "wg_kernels.cuh"

constexpr int BEAM_THREADS = 256;           // scan
constexpr int BEAM_BLOCKS = 4;              // per SM
constexpr int BEAM_WARPS = BEAM_THREADS / 32;
constexpr int BEAM_CHUNK = 512;             // positions per chunk maximum
constexpr uint32_t SCAN_LONG = 4;           // steps of a long item
constexpr uint32_t SCAN_GROUPS = 2;
constexpr int SCAN_COUNTER = 64;            // words from one group's counter to the next
constexpr int PICK_THREADS = 512;
constexpr int PICK_WARPS = PICK_THREADS / 32;
constexpr int PICK_GROUPS = 128;            // at most
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
    uint32_t n_steps;           // of all rows
    uint32_t n_long, n_two;     // items of SCAN_LONG steps, then of two; the rest is dealt step by step
    uint32_t groups, per_group; // of blocks that share a counter
    bool more;                  // there are more items than warps
    Divisor per_row;            // steps of a row
    int32_t chunk_stride;     // chunk maxima per row, a multiple of 4
    int32_t chunk_log2;       // the pick's threads side by side on a row: 32 .. 512
    float *chunk_max;         // [rows][chunk_stride]
    float2 *parts;            // [n_steps] (max, sum) of every step
    int32_t *next_item;       // a counter per group: its items taken beyond the first of every warp; zero between calls
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
    // (what is asked for does not hang on the score: all of it on its way together)
    bool finished;
    if (CTX) {
        const int g = a.gid[row], s = a.sid[row];
        finished = g >= 0 && g < ctx.n_grammars && s > 0 && s == ctx.grammars[g].done;
    } else {
        finished = a.finished && a.finished[row];
    }
    return !(score > -INFINITY) ? BEAM_ROW_DEAD : finished ? BEAM_ROW_FINISHED : BEAM_ROW_LIVE;   // (NaN: dead)
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

// Disallowed elements become -inf, in all pieces of a step.  Byte i of `bits` (fp32: its low nibble)
// belongs to piece i.  bf16: with bit j of every byte moved to the byte's top, one byte permute spreads
// the top bits of two such words over the two elements of a word (its sign-spreading mode, which the
// intrinsic does not know), so a pair costs a permute and a select.
template <int SEL>
__device__ __forceinline__ uint32_t permute(uint32_t lo, uint32_t hi) {
    uint32_t r;
    asm("prmt.b32 %0, %1, %2, %3;" : "=r"(r) : "r"(lo), "r"(hi), "n"(SEL));
    return r;
}

template <typename E, int N>
__device__ __forceinline__ void mask_pieces(uint32_t (&w)[N][4], uint32_t bits) {
    if constexpr (sizeof(E) == 2) {
        static_assert(N == 4, "a byte of bits per piece");
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const uint32_t lo = bits << (7 - 2 * j), hi = bits << (6 - 2 * j);
            const uint32_t keep[4] = {permute<0xCC88>(lo, hi), permute<0xDD99>(lo, hi), permute<0xEEAA>(lo, hi),
                                      permute<0xFFBB>(lo, hi)};
#pragma unroll
            for (int i = 0; i < N; ++i) w[i][j] = (w[i][j] & keep[i]) | (NEG_INF_BF16X2 & ~keep[i]);
        }
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j) w[i][j] = ((bits >> (8 * i + j)) & 1u) ? w[i][j] : NEG_INF_F32;
    }
}

// Largest element of N pieces (NaN elements are passed over).
template <typename E, int N>
__device__ __forceinline__ float pieces_max(const uint32_t (&w)[N][4], int first, int end) {
    if constexpr (sizeof(E) == 2) {
        __nv_bfloat162 m = as_bf162(NEG_INF_BF16X2);
#pragma unroll
        for (int i = 0; i < N; ++i)
            if (i >= first && i < end)
#pragma unroll
                for (int j = 0; j < 4; ++j) m = __hmax2(m, as_bf162(w[i][j]));
        const uint32_t u = bf162_bits(m);
        return fmaxf(__uint_as_float(u << 16), __uint_as_float(u & 0xFFFF0000u));
    } else {
        float m = -INFINITY;
#pragma unroll
        for (int i = 0; i < N; ++i)
            if (i >= first && i < end)
#pragma unroll
                for (int j = 0; j < 4; ++j) m = fmaxf(m, __uint_as_float(w[i][j]));
        return m;
    }
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

// Where a step's exponentials are measured from: 2^(x * log2 e - reference).  Kept in the logarithm's own
// base, so that one fused multiply-add makes the exponent.  m * log2 e is rounded there, by up to |m| * 2^-24,
// and every exponent is off by that, which is put right where the sum is moved.  Beyond |m| = 2^31 or so the sum
// would overflow or vanish first; from 2^20 on the difference x - m is formed instead (finite values that stand
// for a mask, infinities).
constexpr float FAR_M = 1048576.f;

__device__ __forceinline__ float reference(float m) { return __fmul_rn(m, LOG2_E); }

// What the sum of a step with maximum m is multiplied by to be measured from high >= m itself (m = -inf: a sum of
// nothing).
__device__ __forceinline__ float moved(float m, float high) {
    return exp2_fast(fmaf(m - high, LOG2_E, fabsf(m) < FAR_M ? fmaf(-m, LOG2_E, reference(m)) : 0.f));
}

// Two fp32 values in one 64-bit register, for the instructions that work on both.
typedef unsigned long long Pair;
__device__ __forceinline__ Pair pair(float lo, float hi) {
    Pair r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(lo), "f"(hi));
    return r;
}
__device__ __forceinline__ float2 halves(Pair x) {
    float2 r;
    asm("mov.b64 {%0, %1}, %2;" : "=f"(r.x), "=f"(r.y) : "l"(x));
    return r;
}
__device__ __forceinline__ Pair add2(Pair x, Pair y) {
    Pair r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(x), "l"(y));
    return r;
}
__device__ __forceinline__ Pair fma2(Pair x, Pair y, Pair z) {
    Pair r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(x), "l"(y), "l"(z));
    return r;
}

// Adds exp(x - m) of N pieces to two pairs of sums.
template <typename E, int N>
__device__ __forceinline__ void pieces_exp(const uint32_t (&w)[N][4], float m, Pair (&sum)[2]) {
    auto each = [&](auto exponent) {
#pragma unroll
        for (int i = 0; i < N; ++i)
#pragma unroll
            for (int j = 0; j < 4; j += sizeof(E) == 2 ? 1 : 2) {
                const Pair x = sizeof(E) == 2
                    ? pair(__uint_as_float(w[i][j] << 16), __uint_as_float(w[i][j] & 0xFFFF0000u))
                    : pair(__uint_as_float(w[i][j]), __uint_as_float(w[i][(j + 1) & 3]));
                const float2 e = halves(exponent(x));
                Pair &to = sum[sizeof(E) == 2 ? j & 1 : j >> 1];
                to = add2(to, pair(exp2_fast(e.x), exp2_fast(e.y)));
            }
    };
    const Pair scale = pair(LOG2_E, LOG2_E);
    if (fabsf(m) < FAR_M) {                      // uniform
        const Pair minus = pair(-reference(m), -reference(m));
        each([&](Pair x) { return fma2(x, scale, minus); });
    } else {
        const Pair minus = pair(-m, -m), zero = pair(-0.f, -0.f);
        each([&](Pair x) { return fma2(add2(x, minus), scale, zero); });
    }
}

// What (m, s) say of the sum of exp: its logarithm.  (Of one token, whose s is 1 to 2^-22, this is m itself
// from 16 on: a row in a literal keeps its score however long that is.)
__device__ __forceinline__ float log_sum(float m, float s) { return m + logf(s); }

// ---------------------------------------------------------------------------------------
// Scan.  A warp works in steps of 4 KB of one row (eight 16-byte loads per lane, all in flight
// together): 2048 bf16 or 1024 fp32 positions.  Rows differ a lot (a finished one costs nothing, a
// literal state a few sectors, a free-text slot every logit), and so do SMs: with equal shares the
// first was done after 27 us and the last after 58.  So warps take their steps from a counter.
// Additions to one address pass at about 1 per ns, which single steps would be held up by (1024 rows x
// 128256: 68 us), and long items end unevenly; so the items shrink, from four steps to two to one, and
// two halves of the grid, each with a block or more on every SM, have a counter of their own.  No warp
// waits for another (blocks that took eight steps together: 40 us instead of 37 on 512 misaligned rows
// x 151937 summed whole).
//
// Measured with the pick behind it: 47.2 us for 1024 rows x 128256 bf16 (229 MB; the scan itself about
// 43, 5.3 TB/s), 37 us for 512 x 151937 (136 MB), 18 us for 128 x 256000 fp32 of which most are in
// literals, 8.4 us for 32 rows in literals.  What bounds it: 490 instructions a step (the mean over the first
// case's rows, a fifth of which count nothing; about 600 in a step that counts, 250 of them the
// exponentials, 70 the mask) in 32 warps per SM, beside the memory; without exponentials and masks the
// same walk streams at the memory's rate.  More loads in flight did not help where it cost registers or
// instructions: rings in shared memory 53 to 60 us, loads a turn ahead at 80 registers 59, three blocks
// per SM 54.
// ---------------------------------------------------------------------------------------
template <typename E>
struct ScanShape {
    static constexpr int EPC = ElemTraits<E>::PER_CHUNK;
    static constexpr int HALF = 4;                              // loads a mask register covers
    static constexpr int LOADS = 2 * HALF;                      // per lane and step
    static constexpr int STEP = LOADS * 32 * EPC;               // positions: 2048, 1024
    static constexpr int CHUNKS = STEP / BEAM_CHUNK;            // 4, 2
    static constexpr int PER_CHUNK = LOADS / CHUNKS;            // loads per chunk: 2, 4
    static constexpr int WORDS = STEP / 32 / 32;                // mask words per lane and step: 2, 1
};

// The top bit of every byte of x that is not zero (a byte's low bits carry into it, or it is set).
__device__ __forceinline__ uint32_t filled(uint32_t x) { return (((x & 0x7F7F7F7Fu) + 0x7F7F7F7Fu) | x) & 0x80808080u; }

// A row as the scan walks it.
template <typename E, int NORM, bool CTX>
struct ScanRow {
    using S = ScanShape<E>;
    RowView<E> x;
    MaskSource mask;

    __device__ __forceinline__ ScanRow(const BeamArgs &a, const CtxDev &ctx, int row)
        : x(a.logits, a.row_stride, row, a.V), mask(mask_source<CTX>(a, ctx, row)) {}

    // whether step s lies wholly inside the row
    __device__ __forceinline__ bool whole(int s) const {
        return s * S::STEP >= x.off && (s + 1) * S::STEP <= x.V + x.off;
    }

    // lane l: the mask bits of positions 32 * l .. of step s, and of those 1024 further on
    __device__ __forceinline__ void words(uint32_t (&word)[S::WORDS], int s) const {
        const int w = s * (S::STEP / 32) + (int)(threadIdx.x & 31);
        if (whole(s) && (!CTX || !mask.hdr)) {
#pragma unroll
            for (int i = 0; i < S::WORDS; ++i) {
                word[i] = mask.words ? __ldg(mask.words + w + 32 * i) : 0xFFFFFFFFu;
                if (x.off != 0 && mask.words)
                    word[i] = __funnelshift_l(__ldg(mask.words + max(w + 32 * i - 1, 0)), word[i], x.off);
            }
        } else {
#pragma unroll
            for (int i = 0; i < S::WORDS; ++i) word[i] = shifted_word(mask, w + 32 * i, x.off);
        }
    }

    // The step's words dealt to the lanes that hold the elements: byte i of bits[h] (fp32: its low
    // nibble) belongs to this lane's piece HALF * h + i.
    __device__ __forceinline__ static void deal(const uint32_t (&word)[S::WORDS], uint32_t (&bits)[2]) {
        const int lane = threadIdx.x & 31;
        const int byte = lane * S::EPC / 8 & 3;
        const uint32_t pick = byte | (4 + byte) << 4;    // the wanted byte of two words, side by side
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            uint32_t w[S::HALF];
#pragma unroll
            for (int i = 0; i < S::HALF; ++i)
                w[i] = __shfl_sync(0xFFFFFFFFu, word[S::WORDS == 2 ? h : 0],
                                   ((S::WORDS == 2 ? i : h * S::HALF + i) * 32 + lane) * S::EPC / 32);
            bits[h] = __byte_perm(__byte_perm(w[0], w[1], pick), __byte_perm(w[2], w[3], pick), 0x5410);
            if (sizeof(E) == 4) bits[h] = (bits[h] >> (lane * S::EPC & 4)) & 0x0F0F0F0Fu;
        }
    }

    // This lane's pieces of step s.  A piece without an allowed element is not read, unless all are
    // summed: what is left in v is masked later.
    __device__ __forceinline__ void load(uint32_t (&v)[2][S::HALF][4], int s, const uint32_t (&bits)[2]) const {
        const int p = s * S::STEP + (int)(threadIdx.x & 31) * S::EPC;
        if (whole(s)) {
            const E *at = x.base + p;
            if (NORM == WG_BEAM_NORM_FULL || __all_sync(0xFFFFFFFFu, (filled(bits[0]) & filled(bits[1])) == 0x80808080u)) {
#pragma unroll
                for (int h = 0; h < 2; ++h)
#pragma unroll
                    for (int i = 0; i < S::HALF; ++i)
                        asm volatile("ld.global.L1::no_allocate.v4.u32 {%0, %1, %2, %3}, [%4];"
                                     : "=r"(v[h][i][0]), "=r"(v[h][i][1]), "=r"(v[h][i][2]), "=r"(v[h][i][3])
                                     : "l"(at + (h * S::HALF + i) * 32 * S::EPC));
            } else {
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int i = 0; i < S::HALF; ++i)
                    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %5, 0;\n\t"
                                 "@p ld.global.L1::no_allocate.v4.u32 {%0, %1, %2, %3}, [%4];\n\t}"
                                 : "+r"(v[h][i][0]), "+r"(v[h][i][1]), "+r"(v[h][i][2]), "+r"(v[h][i][3])
                                 : "l"(at + (h * S::HALF + i) * 32 * S::EPC),
                                   "r"(bits[h] & (0xFFu << (8 * i))));
            }
        } else {
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int i = 0; i < S::HALF; ++i)
                    if (NORM == WG_BEAM_NORM_FULL || (bits[h] & (0xFFu << (8 * i)))) {
                        const uint4 one = x.piece(p + (h * S::HALF + i) * 32 * S::EPC);
                        v[h][i][0] = one.x; v[h][i][1] = one.y; v[h][i][2] = one.z; v[h][i][3] = one.w;
                    }
        }
    }
};

// Maxima pass over NaN, so a step that counts nothing but -inf and NaN has a maximum of -inf, and no
// exponentials are formed.  Where there is a NaN among them (what is not -inf, then), it goes into the sum,
// and from there into the row's: times what moves it to another maximum it is NaN still.
template <typename E, int N>
__device__ __forceinline__ void keep_nan(const uint32_t (&v)[2][N][4], Pair (&sum)[2]) {
    constexpr uint32_t NOTHING = sizeof(E) == 2 ? NEG_INF_BF16X2 : NEG_INF_F32;
    uint32_t other = 0u;
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int i = 0; i < N; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j) other |= v[h][i][j] ^ NOTHING;
    if (__any_sync(0xFFFFFFFFu, other != 0u)) sum[0] = pair(__int_as_float(0x7FC00000), 0.f);
}

// One step's share of a row: its chunk maxima out, and m, the maximum of what is counted (the same in all
// lanes; -inf coming in), with this lane's sums of exp(x - m) (zero coming in).
template <typename E, int NORM>
__device__ __forceinline__ void scan_step(uint32_t (&v)[2][ScanShape<E>::HALF][4], const uint32_t (&bits)[2],
                                          float *chunks, float &m, Pair (&sum)[2]) {
    using S = ScanShape<E>;
    constexpr uint32_t ALL = sizeof(E) == 2 ? 0xFFFFFFFFu : 0x0F0F0F0Fu;
    constexpr int PER_HALF = S::CHUNKS / 2;
    float best[S::CHUNKS];
#pragma unroll
    for (int i = 0; i < S::CHUNKS; ++i) best[i] = -INFINITY;
    if (NORM == WG_BEAM_NORM_FULL) {
        // the whole vocabulary is summed; the maxima are those of what is allowed
        m = warp_max(fmaxf(pieces_max<E>(v[0], 0, S::HALF), pieces_max<E>(v[1], 0, S::HALF)));
        if (m > -INFINITY) {
            pieces_exp<E>(v[0], m, sum);
            pieces_exp<E>(v[1], m, sum);
        } else {
            keep_nan<E>(v, sum);
        }
    }
    if (__any_sync(0xFFFFFFFFu, (bits[0] | bits[1]) != 0u)) {
        if (!__all_sync(0xFFFFFFFFu, (bits[0] & bits[1]) == ALL)) {
            mask_pieces<E>(v[0], bits[0]);
            mask_pieces<E>(v[1], bits[1]);
        }
#pragma unroll
        for (int i = 0; i < S::CHUNKS; ++i) {
            const int at = i % PER_HALF * S::PER_CHUNK;
            best[i] = warp_max(pieces_max<E>(v[i / PER_HALF], at, at + S::PER_CHUNK));
        }
        if (NORM == WG_BEAM_NORM_ALLOWED) {
            m = best[0];
#pragma unroll
            for (int i = 1; i < S::CHUNKS; ++i) m = fmaxf(m, best[i]);
            if (m > -INFINITY) {
                pieces_exp<E>(v[0], m, sum);
                pieces_exp<E>(v[1], m, sum);
            } else {
                keep_nan<E>(v, sum);
            }
        }
    }
    if ((threadIdx.x & 31) == 0) {
        if constexpr (S::CHUNKS == 4) *reinterpret_cast<float4 *>(chunks) = make_float4(best[0], best[1], best[2], best[3]);
        else *reinterpret_cast<float2 *>(chunks) = make_float2(best[0], best[1]);
    }
}

// A step's results out: of one that allows something (or is summed whole), and of one that does not.
template <typename E, int NORM>
__device__ __forceinline__ void end_step(const BeamArgs &a, int row, int s, bool any,
                                         uint32_t (&v)[2][ScanShape<E>::HALF][4], const uint32_t (&bits)[2]) {
    using S = ScanShape<E>;
    const int lane = threadIdx.x & 31;
    if (!any) {
        if (lane < S::CHUNKS) a.chunk_max[(int64_t)row * a.chunk_stride + s * S::CHUNKS + lane] = -INFINITY;
        if (NORM != WG_BEAM_NORM_NONE && lane == 0)
            a.parts[(uint32_t)row * a.per_row.d + s] = make_float2(-INFINITY, 0.f);
        return;
    }
    float m = -INFINITY;
    Pair sum[2] = {0ull, 0ull};
    scan_step<E, NORM>(v, bits, a.chunk_max + (int64_t)row * a.chunk_stride + s * S::CHUNKS, m, sum);
    if (NORM != WG_BEAM_NORM_NONE) {
        const float2 two = halves(add2(sum[0], sum[1]));
        float total = two.x + two.y;
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) total += __shfl_xor_sync(0xFFFFFFFFu, total, o);
        if (lane == 0) a.parts[(uint32_t)row * a.per_row.d + s] = make_float2(m, total);
    }
}

// What a warp knows of its next step: where it is, and, asked for a turn ahead, its mask words and
// whether the row counts.
template <typename E>
struct ScanNext {
    int row, s;
    uint32_t word[ScanShape<E>::WORDS];
    float score;
    int32_t finished;
};

template <typename E, int NORM, bool CTX>
__global__ void __launch_bounds__(BEAM_THREADS, BEAM_BLOCKS)
beam_scan_kernel(BeamArgs a, CtxDev ctx) {
    using S = ScanShape<E>;
    using Row = ScanRow<E, NORM, CTX>;
    pdl_enter();
    const int lane = threadIdx.x & 31;
    const uint32_t group = blockIdx.x / a.per_group, n_warps = a.per_group * BEAM_WARPS;
    uint32_t step, end;                     // the step that is looked at next, and where its item ends
    const auto item_of = [&](uint32_t nth) {
        const uint32_t item = nth * a.groups + group, two = item - a.n_long, one = two - a.n_two;
        if (item < a.n_long) step = SCAN_LONG * item, end = step + SCAN_LONG;
        else if (two < a.n_two) step = SCAN_LONG * a.n_long + 2 * two, end = step + 2;
        else step = SCAN_LONG * a.n_long + 2 * a.n_two + one, end = step + 1;
    };
    const auto look = [&]() -> ScanNext<E> {
        ScanNext<E> n;
        n.row = -1;
#pragma unroll
        for (int i = 0; i < S::WORDS; ++i) n.word[i] = 0u;
        if (step >= a.n_steps) return n;
        n.row = (int)a.per_row.quotient(step);
        n.s = (int)(step - n.row * a.per_row.d);
        n.score = a.score[n.row];
        n.finished = !CTX && a.finished ? a.finished[n.row] : 0;
        Row(a, ctx, n.row).words(n.word, n.s);
        return n;
    };
    item_of((blockIdx.x - group * a.per_group) * BEAM_WARPS + (threadIdx.x >> 5));
    ScanNext<E> n = look();
    uint32_t v[2][S::HALF][4] = {};
#pragma unroll 1
    while (n.row >= 0) {
        const bool need = ++step == end;
        uint32_t taken = n_warps;
        if (need && a.more && lane == 0) taken += (uint32_t)atomicAdd(a.next_item + group * SCAN_COUNTER, 1);
        const int row = n.row, s = n.s;
        const bool live = CTX ? beam_row_kind<CTX>(a, ctx, row, n.score) == BEAM_ROW_LIVE
                              : n.score > -INFINITY && !n.finished;
        // (most steps of a state inside a literal allow nothing)
        const bool any = NORM == WG_BEAM_NORM_FULL || __any_sync(0xFFFFFFFFu, (n.word[0] | n.word[S::WORDS - 1]) != 0u);
        uint32_t bits[2];
        if (live && any) {
            Row::deal(n.word, bits);
            Row(a, ctx, row).load(v, s, bits);
        }
        if (need) item_of(__shfl_sync(0xFFFFFFFFu, taken, 0));
        n = look();
        if (live) end_step<E, NORM>(a, row, s, any, v, bits);
    }
}

// ---------------------------------------------------------------------------------------
// Pick.  One block per request.  A few KB are read, so it is a chain of latencies, about 4.5 us behind the
// scan whether for one request of 4 beams or for 128 of 8: the rows' facts (with the log-sums of the
// steps' parts), the chunks' scores, a bound that n_out of them reach, the list of those above it and its
// ranks; then the elements of the chosen chunks the same way.  The bound is the n_out-th largest of 16 to
// 128 group maxima, at least twice n_out of them: it lets through little more than n_out, so that every
// listed candidate can be ranked against all others by one thread (no sort, no histogram).  Scores stay
// floats until a candidate is listed (4 beams x 32000 fp32: 8.2 -> 6.5 us a call).  A block that
// finishes last in the scan picking for its request was slower (6.5 -> 7.9 us; 8 requests of 4 beams:
// 9.0 -> 10.6): it comes after a fence and an atomic, where the second launch is already waiting.
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
    // two lists of candidates (chunks, then elements), zero behind the last one
    alignas(16) unsigned long long list[2][PICK_LIST];
    alignas(16) float group[PICK_GROUPS];
    uint32_t chunk[WG_BEAM_MAX_OUT];       // the chosen chunks
    int32_t parent[WG_BEAM_MAX_OUT], token[WG_BEAM_MAX_OUT];
    float score[WG_BEAM_MAX_BEAMS], lse[WG_BEAM_MAX_BEAMS];
    int32_t kind[WG_BEAM_MAX_BEAMS];
    int32_t n_written[WG_BEAM_MAX_BEAMS];  // chunk maxima the scan wrote for the row (0: not live)
    MaskSource mask[WG_BEAM_MAX_BEAMS];
    float bound[2];                        // scores that n_out candidates reach: chunks, elements
    int32_t n[2];
    int32_t digit[256], found_digit, found_above, found_upto;
};

// Calls f(rank, packed key) for the listed candidates of rank below n_out (0 = the largest).
template <typename F>
__device__ __forceinline__ void ranked(const PickShared &sh, int which, int n, int n_out, const F &f) {
    if ((int)threadIdx.x >= n) return;
    const unsigned long long mine = sh.list[which][threadIdx.x];
    int rank = 0;
    for (int j = 0; j < n; j += 8) {       // (the list is a multiple of 8 long, zeros at its end)
#pragma unroll
        for (int u = 0; u < 8; u += 2) {
            const ulonglong2 two = *reinterpret_cast<const ulonglong2 *>(&sh.list[which][j + u]);
            rank += (two.x > mine) + (two.y > mine);
        }
    }
    if (rank < n_out) f(rank, mine);
}
static_assert(PICK_LIST == PICK_THREADS, "a thread per listed candidate");

// sh.bound[0] = the n_out-th largest of the maxima (every thread's `top`) of some groups of threads, a lower
// bound for the n_out-th largest of all: each group's maximum is one of them.  At least twice as many
// groups as are wanted: few of the best then share a group, and few more than n_out reach the bound.
__device__ __forceinline__ void group_bound(PickShared &sh, float top, int n_out) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int per_warp = n_out <= 8 ? 1 : n_out <= 16 ? 2 : n_out <= 32 ? 4 : 8, n_groups = per_warp * PICK_WARPS;
    if (per_warp == 1) top = warp_max(top);
    else for (int o = 16 / per_warp; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, o));
    if ((lane & (32 / per_warp - 1)) == 0) sh.group[warp * per_warp + lane / (32 / per_warp)] = top;
    __syncthreads();
    if ((int)threadIdx.x < n_groups) {
        const float mine = sh.group[threadIdx.x];
        int rank = 0;
#pragma unroll 2
        for (int j = 0; j < n_groups; j += 4) {
            const float4 g = *reinterpret_cast<const float4 *>(&sh.group[j]);
            const int t = (int)threadIdx.x - j;
            rank += (g.x > mine || (g.x == mine && 0 < t)) + (g.y > mine || (g.y == mine && 1 < t)) +
                    (g.z > mine || (g.z == mine && 2 < t)) + (g.w > mine || (g.w == mine && 3 < t));
        }
        if (rank == n_out - 1) sh.bound[0] = mine;
    }
    __syncthreads();
}

// Puts the candidates that `each` enumerates into the (empty) list: those whose score reaches `bound` (and
// is above -inf).  Where they are more than it holds, the bound is raised to that of the candidates' own
// group maxima; where it is overrun still (hosts of equal scores), the packed keys' value that at least
// n_out of them reach and no more than the list holds is found digit by digit.  `each(f)` calls
// f(score, index) for the calling thread's share; no two candidates have an index in common.  Returns how
// many are listed, at least n_out of the best if there are so many.  (Where a request has fewer chunks than
// n_out, its elements come here without a bound: 4 x 16 beams x 1000, 32 results: 22 us; 64 bits found
// one by one: 108.)
template <typename Each>
__device__ __forceinline__ int collect(PickShared &sh, int which, float bound, int n_out, const Each &each) {
    const auto push = [&](float s, uint32_t idx) {
        const int at = atomicAdd(&sh.n[which], 1);
        if (at < PICK_LIST) sh.list[which][at] = pack_key(score_key(s), idx);
    };
    each([&](float s, uint32_t idx) { if (s >= bound && s > -INFINITY) push(s, idx); });
    __syncthreads();
    if (__builtin_expect(sh.n[which] <= PICK_LIST, 1)) return sh.n[which];
    enum { RAISE, PUSH, COUNT, PUSH_FROM_CUT } mode = RAISE;
    unsigned long long cut = 0ull;         // its digits above `shift` are known
    int shift = 56, above = 0;             // keys beyond the known digits
#pragma unroll 1
    while (true) {
        __syncthreads();                   // everybody has read what is cleared now
        if (threadIdx.x < 256) sh.digit[threadIdx.x] = 0;
        for (int i = threadIdx.x; i < PICK_LIST; i += PICK_THREADS) sh.list[which][i] = 0ull;
        if (threadIdx.x == 0) sh.n[which] = 0;
        __syncthreads();
        float top = -INFINITY;
        each([&](float s, uint32_t idx) {
            if (mode == RAISE) {
                top = fmaxf(top, s);
                return;
            }
            if (!(s >= bound && s > -INFINITY)) return;
            const unsigned long long k = pack_key(score_key(s), idx);
            if (mode == COUNT) {
                if (shift == 56 || (k ^ cut) >> (shift + 8) == 0ull) atomicAdd(&sh.digit[k >> shift & 255u], 1);
            } else if (k >= cut) {
                push(s, idx);
            }
        });
        __syncthreads();
        if (mode == RAISE) {
            group_bound(sh, top, n_out);
            bound = fmaxf(bound, sh.bound[0]);
            mode = PUSH;
        } else if (mode != COUNT) {
            if (sh.n[which] <= PICK_LIST) return sh.n[which];
            mode = COUNT;                  // only after the raised bound: the cut leaves no more than fit
        } else {
            // the digit that the n_out-th largest key has, by warp 0 with eight of them to a lane
            if (threadIdx.x < 32) {
                int mine = 0;
                for (int i = 0; i < 8; ++i) mine += sh.digit[255 - (int)threadIdx.x * 8 - i];
                int upto = mine;
#pragma unroll
                for (int o = 1; o < 32; o <<= 1) {
                    const int y = __shfl_up_sync(0xFFFFFFFFu, upto, o);
                    if ((int)threadIdx.x >= o) upto += y;
                }
                if (above + upto >= n_out && above + upto - mine < n_out) {
                    int before = above + upto - mine, d = 255 - (int)threadIdx.x * 8;
                    while (before + sh.digit[d] < n_out) before += sh.digit[d--];
                    sh.found_digit = d;
                    sh.found_above = before;
                    sh.found_upto = before + sh.digit[d];
                }
            }
            __syncthreads();
            cut |= (unsigned long long)sh.found_digit << shift;
            above = sh.found_above;
            if (sh.found_upto <= PICK_LIST) mode = PUSH_FROM_CUT;   // (at the last digit it is: keys differ)
            else shift -= 8;
        }
    }
}

// The request's best candidates, listed in sh.list[1]: the n_out best and possibly more.  Returns how
// many are listed.
template <typename E, bool CTX>
__device__ __forceinline__ int beam_pick(PickShared &sh, const BeamArgs &a, const CtxDev &ctx, int req) {
    constexpr int EPC = ElemTraits<E>::PER_CHUNK;
    constexpr int PER_CHUNK = BEAM_CHUNK / (32 * EPC);
    constexpr int HELD = 8;                // chunk maxima a thread keeps in registers
    constexpr int PARTS = 4;               // pairs a lane has in flight
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int K = a.n_beam, row0 = req * K;
    const int n_chunks = a.chunk_stride;
    // A thread's chunks: column c0, c0 + width, .. of beam b0, b0 + side, ..  They are asked for before
    // anything else is known, so that their latency passes together with that of the rows' facts.
    const int width = 1 << a.chunk_log2, side = PICK_THREADS >> a.chunk_log2;
    const int c0 = threadIdx.x & (width - 1), b0 = threadIdx.x >> a.chunk_log2;
    const int turns = (n_chunks + width - 1) >> a.chunk_log2;           // columns of a thread on a row
    const int slots = (K + side - 1) / side * turns;
    const float *maxima = a.chunk_max + (int64_t)row0 * n_chunks;
    // calls f(slot, beam, column) for the thread's slots [first, end)
    const auto visit = [&](int first, int end, auto f) {
        int b = b0 + first / turns * side, turn = first % turns;
        for (int j = first; j < end; ++j) {
            f(j, b, c0 + (turn << a.chunk_log2));
            if (++turn == turns) {
                turn = 0;
                b += side;
            }
        }
    };
    float held[HELD];
    {
        int b = b0, turn = 0;
#pragma unroll
        for (int j = 0; j < HELD; ++j) {
            const int c = c0 + (turn << a.chunk_log2);
            held[j] = -INFINITY;
            if (j < slots && b < K && c < n_chunks) held[j] = maxima[b * n_chunks + c];
            if (++turn == turns) {
                turn = 0;
                b += side;
            }
        }
    }
    sh.list[0][threadIdx.x] = sh.list[1][threadIdx.x] = 0ull;
    if (threadIdx.x < 2) sh.n[threadIdx.x] = 0;
    if (threadIdx.x == 2) sh.bound[0] = sh.bound[1] = -INFINITY;
    // ---- the rows: whether they count, and their log-sum-exp from the steps' pairs (those of a row that
    // does not count are left over: read all the same, in one go with the rest, and not used)
    for (int b = warp; b < K; b += PICK_WARPS) {
        const int row = row0 + b, n_parts = (int)a.per_row.d;
        const float2 *parts = a.parts + (int64_t)row * n_parts;
        const bool sums = a.norm != WG_BEAM_NORM_NONE;
        const float score = a.score[row];
        float2 p[PARTS];
#pragma unroll
        for (int i = 0; i < PARTS; ++i) {
            p[i] = make_float2(-INFINITY, 0.f);
            if (sums && lane + 32 * i < n_parts) p[i] = parts[lane + 32 * i];
        }
        const int kind = beam_row_kind<CTX>(a, ctx, row, score);
        float lse = 0.f;
        if (sums) {
            float m = p[0].x, s = 0.f;
#pragma unroll
            for (int i = 1; i < PARTS; ++i) m = fmaxf(m, p[i].x);
            for (int i = lane + 32 * PARTS; i < n_parts; i += 32) m = fmaxf(m, parts[i].x);
            m = warp_max(m);
            if (m > -INFINITY) {           // (a pair that saw nothing is (-inf, 0))
#pragma unroll
                for (int i = 0; i < PARTS; ++i) s += p[i].y * moved(p[i].x, m);
                for (int i = lane + 32 * PARTS; i < n_parts; i += 32) s += parts[i].y * moved(parts[i].x, m);
            }
#pragma unroll
            for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xFFFFFFFFu, s, o);
            lse = log_sum(m, s);
        }
        if (lane == 0) {
            const RowView<E> x(a.logits, a.row_stride, row, a.V);
            sh.score[b] = score;
            sh.lse[b] = lse;
            sh.kind[b] = kind;
            sh.n_written[b] = kind == BEAM_ROW_LIVE ? (a.V + x.off + BEAM_CHUNK - 1) / BEAM_CHUNK : 0;
            sh.mask[b] = mask_source<CTX>(a, ctx, row);
        }
    }
    __syncthreads();
    // ---- the n_out best chunks
    const auto chunk_score = [&](int b, int c, float maximum) -> float {
        return b < K && c < sh.n_written[b] ? sh.score[b] + (maximum - sh.lse[b]) : -INFINITY;
    };
    float top = -INFINITY;
    {
        int b = b0, turn = 0;
#pragma unroll
        for (int j = 0; j < HELD; ++j) {
            if (j >= slots) break;                 // uniform
            held[j] = chunk_score(b, c0 + (turn << a.chunk_log2), held[j]);
            top = fmaxf(top, held[j]);
            if (++turn == turns) {
                turn = 0;
                b += side;
            }
        }
    }
    const auto beyond = [&](int b, int c) -> float {               // a chunk that is not held
        return b < K && c < n_chunks ? chunk_score(b, c, maxima[b * n_chunks + c]) : -INFINITY;
    };
    visit(HELD, slots, [&](int, int b, int c) { top = fmaxf(top, beyond(b, c)); });
    group_bound(sh, top, a.n_out);
    int n = collect(sh, 0, sh.bound[0], a.n_out, [&](auto f) {
        int b = b0, turn = 0;
#pragma unroll
        for (int j = 0; j < HELD; ++j) {
            if (j >= slots) break;
            f(held[j], (uint32_t)(b * n_chunks + c0 + (turn << a.chunk_log2)));
            if (++turn == turns) {
                turn = 0;
                b += side;
            }
        }
        visit(HELD, slots, [&](int, int bb, int c) { f(beyond(bb, c), (uint32_t)(bb * n_chunks + c)); });
    });
    ranked(sh, 0, n, a.n_out, [&](int rank, unsigned long long k) {
        sh.chunk[rank] = 0xFFFFFFFFu - (uint32_t)k;
        if (rank == a.n_out - 1) sh.bound[1] = key_score((uint32_t)(k >> 32));   // n_out elements reach this
    });
    __syncthreads();
    // ---- the n_out best elements of those chunks, and the finished rows' candidates
    // (a warp takes 32 pieces of a chunk at a time)
    const int n_sel = min(n, a.n_out) * PER_CHUNK;
    return collect(sh, 1, sh.bound[1], a.n_out, [&](auto f) {
        for (int i = warp; i < n_sel; i += PICK_WARPS) {
            const int at = (int)sh.chunk[i / PER_CHUNK];
            const int b = at / n_chunks, p = (at - b * n_chunks) * BEAM_CHUNK + (i % PER_CHUNK * 32 + lane) * EPC;
            const RowView<E> x(a.logits, a.row_stride, row0 + b, a.V);
            const uint4 u = x.piece(p);
            uint32_t bits = shifted_word(sh.mask[b], p >> 5, x.off) >> (p & 31);
            const float score = sh.score[b], lse = sh.lse[b];
            const uint32_t v[4] = {u.x, u.y, u.z, u.w};
            const uint32_t idx = (uint32_t)b * (uint32_t)a.V + (uint32_t)(p - x.off);
#pragma unroll
            for (int j = 0; j < EPC; ++j) {
                const uint32_t e = sizeof(E) == 2
                    ? ((j & 1) ? (v[j >> 1] & 0xFFFF0000u) : (v[j >> 1] << 16)) : v[j & 3];
                f((bits >> j) & 1u ? score + (__uint_as_float(e) - lse) : -INFINITY, idx + j);
            }
        }
        if ((int)threadIdx.x < K && sh.kind[threadIdx.x] == BEAM_ROW_FINISHED)
            f(sh.score[threadIdx.x], threadIdx.x * (uint32_t)a.V + (uint32_t)a.eos);
    });
}

// With a context the selection writes grammar ids, which the kernels of a step that follows read ahead of
// their wait: dependents start at its end then.
template <bool CTX>
__device__ __forceinline__ void select_enter() {
    if constexpr (CTX) pdl_wait();
    else pdl_enter();
}

// The request's selection out and, with a context, its states moved on.
template <typename E, bool CTX>
__device__ __forceinline__ void select_request(PickShared &sh, const BeamArgs &a, const CtxDev &ctx, const VocabDev &v,
                                               const BeamStepArgs &st, int req, float *score_out, int32_t *parent_out,
                                               int32_t *token_out) {
    const int n = beam_pick<E, CTX>(sh, a, ctx, req);
    // ---- out, best first
    const int64_t out0 = (int64_t)req * a.n_out;
    if ((int)threadIdx.x < a.n_out && (int)threadIdx.x >= n) {
        score_out[out0 + threadIdx.x] = -INFINITY;
        parent_out[out0 + threadIdx.x] = sh.parent[threadIdx.x] = -1;
        token_out[out0 + threadIdx.x] = sh.token[threadIdx.x] = -1;
    }
    ranked(sh, 1, n, a.n_out, [&](int rank, unsigned long long k) {
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

template <typename E, bool CTX>
__global__ void __launch_bounds__(PICK_THREADS)
beam_pick_kernel(BeamArgs a, CtxDev ctx, VocabDev v, BeamStepArgs st, float *score_out,
                 int32_t *parent_out, int32_t *token_out) {
    __shared__ PickShared sh;
    select_enter<CTX>();
    if (blockIdx.x == 0 && threadIdx.x < a.groups) a.next_item[threadIdx.x * SCAN_COUNTER] = 0;
    select_request<E, CTX>(sh, a, ctx, v, st, blockIdx.x, score_out, parent_out, token_out);
}

__device__ __forceinline__ void cluster_sync() {
    asm volatile("barrier.cluster.arrive.aligned;\n\tbarrier.cluster.wait.aligned;" ::: "memory");
}

// Both in one launch, for few requests: a cluster per request, large enough that every step of its rows has
// a warp; the cluster's first block picks.  On the device it takes what two launches take (1 x 4 beams x
// 32000 fp32: 6.6 us; the cluster's start and barrier are as long as the overlapped second launch), and the
// host is done 2.5 us earlier.  With a second step for a warp it lost (8 x 4 beams x 128256: 9.9 us
// instead of 8.4).
constexpr int SMALL_CLUSTER = 16;           // blocks, at most

template <typename E, int NORM, bool CTX>
__global__ void __launch_bounds__(PICK_THREADS)
beam_small_kernel(BeamArgs a, CtxDev ctx, VocabDev v, BeamStepArgs st, float *score_out,
                  int32_t *parent_out, int32_t *token_out) {
    using S = ScanShape<E>;
    using Row = ScanRow<E, NORM, CTX>;
    __shared__ PickShared sh;
    select_enter<CTX>();
    const int i = blockIdx.x * PICK_WARPS + (threadIdx.x >> 5);
    const int b = (int)a.per_row.quotient((uint32_t)i), s = i - b * (int)a.per_row.d, row = blockIdx.y * a.n_beam + b;
    if (b < a.n_beam) {
        const float score = a.score[row];
        uint32_t word[S::WORDS], bits[2], x[2][S::HALF][4] = {};
        Row(a, ctx, row).words(word, s);
        if (beam_row_kind<CTX>(a, ctx, row, score) == BEAM_ROW_LIVE) {
            const bool any = NORM == WG_BEAM_NORM_FULL || __any_sync(0xFFFFFFFFu, (word[0] | word[S::WORDS - 1]) != 0u);
            if (any) {
                Row::deal(word, bits);
                Row(a, ctx, row).load(x, s, bits);
            }
            end_step<E, NORM>(a, row, s, any, x, bits);
        }
    }
    cluster_sync();
    if (blockIdx.x == 0) select_request<E, CTX>(sh, a, ctx, v, st, blockIdx.y, score_out, parent_out, token_out);
}

// ---------------------------------------------------------------------------------------
// Back-track.  The walk from the last step to the first is a chain of dependent look-ups, so the steps are
// cut into segments: every segment is first walked from all beams at once (a map from its last beams
// to its first), the maps are composed, and then every segment is walked again from the beam that each
// final beam really comes by.  A cluster of up to eight blocks takes a group of neighbouring requests (as many
// as make up to 32 columns: 128 bytes of every step, read in whole lines) and a tile of steps, a part of the
// tile for each block; the parts' maps are exchanged through the cluster's shared memory.  Within a
// block a thread walks one column of one of the part's segments.
//
// Measured: 4.2 us for 256 steps of 8 x 4; for 4096 steps of 128 x 8 (50 MB) 17.4 us from memory
// (2.9 TB/s), 12.5 from L2.  Bound by the staging of a part in shared memory and by the two walks' chains of
// look-ups (32 steps each), during which nothing is loaded.  What would load meanwhile cost more than it
// gave: tokens copied past the registers, word by word: 22.7 us; sixteen loads of each array in flight,
// kept across the walks: 19.7 (everything runs once: longer code is fetched for longer, 4.2 -> 7.1 us
// for the small search).  A broken way follows a column of its own instead of being
// tested for at every step (27 -> 13 us).
// ---------------------------------------------------------------------------------------
constexpr int BACK_THREADS = 512;
constexpr int BACK_STEPS = 512;         // most steps of a block's part
constexpr int BACK_CLUSTER = 8;         // most blocks of a cluster
constexpr int BACK_DEAD = 32;           // the column of a way that broke off: it leads to itself, its token is -1
constexpr int BACK_ROW = 33;            // columns of a step (odd: a column's steps lie in different banks)

struct BackShared {
    int32_t token[BACK_STEPS * BACK_ROW];     // [step][column]
    uint8_t parent[BACK_STEPS * BACK_ROW];    // [step][column]: a column of the step before
    uint8_t path[BACK_STEPS * BACK_ROW];      // [step][column]: the step's column that this final one comes by
    uint8_t maps[2][BACK_THREADS / 32 * BACK_ROW];   // [segment][column]
    uint8_t part[BACK_ROW];                   // the whole part's map
    uint8_t at[32], from[32];           // where the final columns stand before the tile; where they enter the part
};

struct BackArgs {
    const int32_t *token, *parent;
    int32_t *out;
    int32_t T, n_req, K;
    int32_t group;                      // requests of a block
    int32_t steps;                      // of a part (at most BACK_STEPS)
};

// The byte at `p` of this block's shared memory, in the shared memory of the cluster's block `rank`.
__device__ __forceinline__ uint32_t cluster_byte(const uint8_t *p, uint32_t rank) {
    uint32_t at, x;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(at) : "r"((uint32_t)__cvta_generic_to_shared(p)), "r"(rank));
    asm volatile("ld.shared::cluster.u8 %0, [%1];" : "=r"(x) : "r"(at) : "memory");
    return x;
}

__global__ void __launch_bounds__(BACK_THREADS, 2)
beam_backtrack_kernel(BackArgs a) {
    extern __shared__ uint8_t back_smem[];
    BackShared &sh = *reinterpret_cast<BackShared *>(back_smem);
    pdl_enter();
    const int n_parts = (int)gridDim.x, part = (int)blockIdx.x;      // the cluster is the grid's x extent
    const int64_t step = (int64_t)a.n_req * a.K;                     // entries per step
    const int64_t col0 = (int64_t)blockIdx.y * a.group * a.K;
    const int width = (int)min((int64_t)a.group * a.K, step - col0);
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;      // a warp per segment, a lane per column
    constexpr int SEGMENTS = BACK_THREADS / 32;
    const bool mine = lane < width;
    const int base = lane / a.K * a.K;                               // the lane's request's first column
    const int tile = n_parts * a.steps;
    if (threadIdx.x < 32) sh.at[threadIdx.x] = (uint8_t)(mine ? lane : BACK_DEAD);
    for (int t = threadIdx.x; t < a.steps; t += BACK_THREADS) {      // (nothing else is written there)
        sh.parent[t * BACK_ROW + BACK_DEAD] = (uint8_t)BACK_DEAD;
        sh.token[t * BACK_ROW + BACK_DEAD] = -1;
    }
    if (threadIdx.x < 2 * SEGMENTS)
        sh.maps[threadIdx.x / SEGMENTS][threadIdx.x % SEGMENTS * BACK_ROW + BACK_DEAD] = (uint8_t)BACK_DEAD;
    for (int t1 = a.T; t1 > 0; t1 -= tile) {                         // tiles from the last to the first
        const int t0 = t1 - tile + part * a.steps;                   // this block's part: [max(t0, 0), t0 + steps)
        const int first = max(t0, 0), n = max(0, t0 + a.steps - first);
        __syncthreads();                                             // the previous tile is done with
        // ---- in: a warp reads a step's line
        {
            constexpr int LOADS = 8;                                 // in flight, of each array
            const int64_t stride = SEGMENTS * step;
            const int64_t at0 = (first + warp) * step + col0 + (mine ? lane : 0);
            const int32_t *parent = a.parent + at0, *token = a.token + at0;
            const uint32_t most = mine ? (uint32_t)a.K : 0u;
            int to = warp * BACK_ROW + lane;
            const auto put = [&](int32_t p, int32_t x) {
                sh.parent[to] = (uint8_t)((uint32_t)p < most ? base + p : BACK_DEAD);
                sh.token[to] = x;
                to += SEGMENTS * BACK_ROW;
            };
            int s = warp;
#pragma unroll 1
            for (; s + (LOADS - 1) * SEGMENTS < n; s += LOADS * SEGMENTS) {
                int32_t p[LOADS], x[LOADS];
#pragma unroll
                for (int i = 0; i < LOADS; ++i, parent += stride, token += stride) {
                    p[i] = __ldcs(parent);
                    x[i] = __ldcs(token);
                }
#pragma unroll
                for (int i = 0; i < LOADS; ++i) put(p[i], x[i]);
            }
#pragma unroll 1
            for (; s < n; s += SEGMENTS, parent += stride, token += stride) put(__ldcs(parent), __ldcs(token));
        }
        __syncthreads();
        // ---- the segments' maps
        const int per = (n + SEGMENTS - 1) / SEGMENTS;
        const int lo = min(n, warp * per), hi = min(n, lo + per);
        int b = lane;
#pragma unroll 4
        for (int t = (hi - 1) * BACK_ROW; t >= lo * BACK_ROW; t -= BACK_ROW) b = sh.parent[t + b];
        sh.maps[0][warp * BACK_ROW + lane] = (uint8_t)b;
        __syncthreads();
        // maps[s] becomes the composition of the maps of all segments from the last down to s
        int now = 0;
#pragma unroll 1
        for (int d = 1; d < SEGMENTS; d <<= 1) {
            if (warp + d < SEGMENTS) b = sh.maps[now][warp * BACK_ROW + sh.maps[now][(warp + d) * BACK_ROW + lane]];
            now ^= 1;
            sh.maps[now][warp * BACK_ROW + lane] = (uint8_t)b;
            __syncthreads();
        }
        // ---- the parts: from the last one down to this one, and on to the first
        if (threadIdx.x < BACK_ROW) sh.part[threadIdx.x] = sh.maps[now][threadIdx.x];
        if (n_parts > 1) cluster_sync();
        else __syncthreads();
        if (threadIdx.x < 32) {
            int c = sh.at[threadIdx.x];
            for (int q = n_parts - 1; q >= 0; --q) {
                if (q == part) sh.from[threadIdx.x] = (uint8_t)c;
                c = (int)cluster_byte(&sh.part[c], (uint32_t)q);
            }
            sh.at[threadIdx.x] = (uint8_t)c;
        }
        if (n_parts > 1) cluster_sync();                             // the maps have been read, and `from` is there
        else __syncthreads();
        // ---- the way
        b = sh.from[lane];
        if (warp + 1 < SEGMENTS) b = sh.maps[now][(warp + 1) * BACK_ROW + b];
#pragma unroll 4
        for (int t = (hi - 1) * BACK_ROW; t >= lo * BACK_ROW; t -= BACK_ROW) {
            sh.path[t + lane] = (uint8_t)b;
            b = sh.parent[t + b];
        }
        __syncthreads();
        // ---- out: a warp writes a column, 32 steps at a time
        for (int c = warp; c < width; c += SEGMENTS) {
            int32_t *out = a.out + (col0 + c) * a.T + first;
            const bool gone = sh.at[c] == BACK_DEAD;                 // it broke off here or further on: no sequence
            const int32_t *token = sh.token + lane * BACK_ROW;
            const uint8_t *path = sh.path + lane * BACK_ROW + c;
            if (gone) {
                for (int t = lane; t < n; t += 32) out[t] = -1;
            } else {
#pragma unroll 4
                for (int t = lane; t < n; t += 32, token += 32 * BACK_ROW, path += 32 * BACK_ROW) out[t] = token[*path];
            }
        }
    }
    // a way back that broke off in a later tile than the first: what was written of it before goes
    __syncthreads();
    if (a.T > tile)
        for (int c = 0; c < width; ++c)
            if (sh.at[c] == BACK_DEAD)
                for (int t = part * BACK_THREADS + (int)threadIdx.x; t < a.T; t += n_parts * BACK_THREADS)
                    a.out[(col0 + c) * a.T + t] = -1;
}
