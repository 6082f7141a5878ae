// Attention of single tokens over a paged cache (wg_kv_attend of wg.h).
//
// The work is memory: every key and value is read once, by one warp, for the handful of rows (a head's queries) that
// need it.  A pair is what one head of a token's keys and values comes to: a run of units, tiles of 16 or 32 positions.  All
// units of a call, in order of tokens and heads, are dealt out in equal contiguous shares, whatever the lengths, to
// warps that work by themselves, or, of pairs that several warps work on together (few pairs; positions that a group of tokens has in
// common), to blocks.  A pair that was cut between shares is joined by a kernel that follows, from partial results in scratch,
// in an order that the lengths (and, of what a group shares, its tables) decide alone.
//
// A warp has a ring of tiles of its own, filled with cp.async, and the usual running maximum and sum: for x =
// scale q.k and the maximum m so far, p = 2^(x - m), l = sum of p, o = sum of p v, all multiplied by 2^(m_old - m) when m
// grows.  Both products are taken transposed, positions by rows and dimensions by rows: the few rows are then the N of
// mma.m16n8k16, which comes in eights, and the keys and values the M.  Scores become the second product's operand by
// transposing 8 x 8 pieces in registers.  Keys and values are read with plain 16-byte loads: the order of a dot product's terms
// is free, so a lane takes eight neighbouring dimensions of a key instead of the instruction's scattered pairs (and the
// queries are loaded the same way), and of the values it takes the same eight dimensions of four positions and pairs
// them with byte permutes, which makes the rows of the result neighbouring dimensions too.
//
// 8-bit caches.  Codes are exact in fp16.  Queries enter in fp16, divided by a power of two per row (a query of 2^-14 of the
// row's largest loses its last bits: 2^-25 of the largest).  A key's scale multiplies the score.  A value's scale s cannot
// simply multiply p, which then might fall below fp16's range while it matters: with x' = x + log2 s and the maximum m taken
// over x', p' = 2^(x' - m) is at most 1 and largest where the result comes from, and l is the sum of 2^(x - m), held 2^12 times as
// large: beside a scale of 2^121, the largest that is written, it has weights down to 2^-17 of the largest, beside 2^100 down to 2^-38.
// For m, scales below 2^-96 count as that, which keeps l below 2^108 a position (where a lane's share of it passes 2^112, m is raised by 8),
// and so do infinities and NaN: the rest of such a scale, or what it is, is put into p' where a tile has some, and the sum, which has no
// values in it, goes without.
// A vector that was written as zeros has the scale 1 and yet no part in the result: where one would raise the maximum it counts as 2^-96 too.
//
// Scores of any size.  A score of 10^7 is rounded to whole numbers in fp32, and so would be x less a rounded maximum, or log2 s
// beside it.  So the maximum is subtracted before anything else is done: with 16 bits m is one of the dot products as they are, and
// p = 2^((x - m) scale) is 1 at m.  With 8 bits x' is made from dot products less an origin, 0 until x' passes 256 and then
// moved to where the scores are, and what is kept of a row comes with its origin (Frame).
#pragma once

#include <type_traits>

#include "wg_cache.cuh"

constexpr int MAX_TOKENS = 384;         // of one launch: their ranges and prefix sums are in shared memory

constexpr int ATTEND_WARPS = 4, ATTEND_THREADS = 32 * ATTEND_WARPS;
constexpr int PART_ROWS = 16 * ATTEND_WARPS;      // rows that a block can work on together

__device__ __forceinline__ int64_t quotient(int64_t a, int64_t b) {      // of numbers >= 0; mostly small ones
    return ((a | b) >> 32) == 0 ? (int64_t)((uint32_t)a / (uint32_t)b) : a / b;
}

// Units of work, dealt out to workers in equal contiguous shares: the first `extra` have base + 1 units, the others base.
struct Deal {
    int64_t base, extra;
    int32_t workers;
    __device__ void make(int64_t units, int32_t n) {
        workers = (int32_t)min((int64_t)n, units);
        base = workers > 0 ? quotient(units, workers) : 0;
        extra = units - base * workers;
    }
    __device__ __forceinline__ int64_t begin(int w) const { return w * base + min((int64_t)w, extra); }
    __device__ __forceinline__ int owner(int64_t unit) const {
        const int64_t larger = extra * (base + 1);
        return unit < larger ? (int)quotient(unit, base + 1) : (int)(extra + quotient(unit - larger, base));
    }
};

// What a launch is about, in shared memory.
struct Book {
    int64_t upto[MAX_TOKENS + 1];         // units of its own before a token
    int64_t shared_upto[MAX_TOKENS + 1];  // shared units before a group
    int32_t seq[MAX_TOKENS], from[MAX_TOKENS], end[MAX_TOKENS];   // a token's own positions: from .. end - 1; end 0: it has no row
    int32_t to[MAX_TOKENS];               // shared positions of a group: 0 .. to - 1 (without groups: from[t] .. to[t] - 1)
    Deal shared, own;                     // the blocks' units, and the warps'
};

struct AttendArgs {
    const uint16_t *q;
    uint16_t *out;
    float *lse;
    int64_t q_stride, out_stride;
    const int32_t *table, *len, *seq, *pos;
    const int64_t *slot;
    int64_t stride;
    int32_t max_blocks, n_seq, n_tokens, window;
    int32_t n_q_heads, rows;      // rows: query heads of a key head
    int32_t group, n_groups;
    int32_t row_blocks;           // of 8 or 16 rows each, of one token and key head
    int32_t together;             // key heads that the warps of a block take side by side: 1, 2 or 4
    int32_t q_bf16;
    float scale;                  // times log2(e)
    // scratch
    int32_t part_rows;            // rows of a warp's partial result
    int32_t *shared;              // [n_groups] positions from 0 on that a group has in the same blocks
    float *block_parts;           // [block][2][PART_ROWS]: partial results of a pair that begins before a block's share, or within
    float *warp_parts;            // [worker][together][2][part_rows]: ... before a share of the warps' work, or within
    float *shared_rows;           // [n_tokens][n_q_heads]: shared results that one block did by itself
    float *own_rows;              // ... and what is to be joined with them
    int2 *shared_cuts, *own_cuts; // of every pair, for the kernel that joins
    // how the kernel is cut out
    int32_t warp_rows, shared_rows_each;  // rows that a warp works for by itself, and those of a shared pair
    int32_t shared_row_blocks;    // 0: there are no pairs for whole blocks
    int32_t grouped, origins;
};

namespace {

constexpr float NEG_INFINITY = -__builtin_huge_valf();

__device__ __forceinline__ void attend_enter() {
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    asm volatile("griddepcontrol.wait;" ::: "memory");
}

// What a token sees: positions first .. end - 1 of sequence s; end = 0: nothing.
struct Seen {
    int32_t s, first, end;
};

__device__ __forceinline__ Seen seen_by(const AttendArgs &a, const CacheDev &cache, int t) {
    Seen r{0, 0, 0};
    if (t >= a.n_tokens) return r;
    int32_t s = t, p;
    if (a.seq) {
        s = a.seq[t];
        p = a.slot[t] < 0 ? -1 : a.pos[t];
    } else {
        p = a.len[t] - 1;
    }
    if (s < 0 || s >= a.n_seq || p < 0 || p == 0x7FFFFFFF || (int64_t)p >= (int64_t)a.max_blocks * cache.block.d) return r;
    r.s = s;
    r.first = a.window > 0 && p >= a.window ? p - a.window + 1 : 0;
    r.end = p + 1;
    return r;
}

// Tiles of `size` positions.
__device__ __forceinline__ int32_t tiles_of(int32_t first, int32_t end, uint32_t size) {
    return first < end ? (int32_t)(((uint32_t)(end - first) + size - 1) / size) : 0;
}

// A block per group of tokens: how far their tables agree.  A token has a say about the columns that it sees.  Latencies: lengths,
// then a round of loads for every four of the group's tables and 128 columns.
__global__ void __launch_bounds__(ATTEND_THREADS)
attend_plan_kernel(const __grid_constant__ CacheDev cache, const __grid_constant__ AttendArgs a) {
    attend_enter();
    __shared__ Seen seen[WG_BEAM_MAX_BEAMS];
    __shared__ int32_t differs;
    const int g = blockIdx.x, t0 = g * a.group;
    if (threadIdx.x == 0) differs = 0x7FFFFFFF;
    if ((int)threadIdx.x < a.group) seen[threadIdx.x] = seen_by(a, cache, t0 + (int)threadIdx.x);
    __syncthreads();
    int leader = -1, end = 0, second = 0;     // the longest token, and how far any other one of another sequence goes
    for (int m = 0; m < a.group; ++m)
        if (seen[m].end > end) leader = m, end = seen[m].end;
    for (int m = 0; m < a.group; ++m)
        if (leader >= 0 && seen[m].s != seen[leader].s) second = max(second, seen[m].end);
    // (a warp takes every fourth token, its lanes four columns each at a time)
    const int cols = second > 0 ? (int)cache.block.quotient((uint32_t)(second - 1)) + 1 : 0;
    const int32_t *mine = a.table + (leader >= 0 ? seen[leader].s * a.stride : 0);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    for (uint32_t c0 = 0; c0 < (uint32_t)cols; c0 += 128) {       // (up to 2^31 columns)
        int at = 0x7FFFFFFF;
        for (int m = warp; m < a.group; m += ATTEND_WARPS) {
            const Seen r = seen[m];
            if (r.end == 0 || r.s == seen[leader].s) continue;
            const uint32_t mine_cols = cache.block.quotient((uint32_t)(r.end - 1)) + 1;
            const int32_t *theirs = a.table + r.s * a.stride;
            int32_t x[4], y[4];
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                const uint32_t c = c0 + u * 32 + lane;
                x[u] = c < mine_cols ? theirs[c] : 0, y[u] = c < mine_cols ? mine[c] : 0;
            }
#pragma unroll
            for (int u = 3; u >= 0; --u)
                if (x[u] != y[u]) at = min(at, (int)(c0 + u * 32 + lane));
        }
        if (at < 0x7FFFFFFF) atomicMin(&differs, at);
        if (__syncthreads_or(at < 0x7FFFFFFF)) break;
    }
    if (threadIdx.x == 0) {
        a.shared[g] = a.window > 0 ? 0 : (int)min((int64_t)end, (int64_t)differs * cache.block.d);
    }
}

// ---- pieces of the inner loop --------------------------------------------------------------------------------

__device__ __forceinline__ uint32_t shared_address(const void *p) { return (uint32_t)__cvta_generic_to_shared(p); }
__device__ __forceinline__ void copy16(uint32_t to, const void *from, bool real) {   // zeros where it is not
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(to), "l"(from), "r"(real ? 16 : 0) : "memory");
}
__device__ __forceinline__ void copy16(uint32_t to, const void *from) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(to), "l"(from) : "memory");
}
__device__ __forceinline__ void copy4(uint32_t to, const void *from, bool real) {
    asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(to), "l"(from), "r"(real ? 4 : 0) : "memory");
}
__device__ __forceinline__ uint4 load16(uint32_t at) {
    uint4 x;
    asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(x.x), "=r"(x.y), "=r"(x.z), "=r"(x.w) : "r"(at) : "memory");
    return x;
}
__device__ __forceinline__ uint2 load8(uint32_t at) {
    uint2 x;
    asm volatile("ld.shared.v2.u32 {%0, %1}, [%2];" : "=r"(x.x), "=r"(x.y) : "r"(at) : "memory");
    return x;
}
__device__ __forceinline__ float power2(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

__device__ __forceinline__ void multiply(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1, __nv_bfloat16) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void multiply(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1, __half) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

__device__ __forceinline__ uint32_t transpose8x8(uint32_t x) {     // of 16-bit elements
    uint32_t y;
    asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
    return y;
}

// KV: what the cache holds; DP: the head size, rounded up (dimensions beyond it are zeros).
template <typename KV, int DP>
struct Shape {
    static constexpr bool NARROW = std::is_same<KV, E4m3>::value || std::is_same<KV, Int8>::value;
    using Mma = typename std::conditional<std::is_same<KV, __nv_bfloat16>::value, __nv_bfloat16, __half>::type;
    static constexpr int BYTES = NARROW ? 1 : 2;
    static constexpr int CHUNKS = DP * BYTES / 16;          // 16-byte pieces of a vector
    static constexpr int TILE = DP * BYTES <= 128 ? 32 : 16;      // positions
    static constexpr int SUBS = TILE / 16;
    static constexpr uint32_t ALL = TILE == 32 ? 0xFFFFFFFFu : 0xFFFFu;
    static constexpr int PLANE = TILE * DP * BYTES;         // a tile of keys, or of values
    static constexpr int STAGE = 2 * PLANE;
    static constexpr int STAGES = 3;
    static constexpr int SMEM = ATTEND_WARPS * STAGES * STAGE;
    static constexpr int BLOCKS = SMEM > 110 * 1024 ? 1 : 2;        // on an SM
    // fp16 weights are 2^15 times as large as they need be (and so are results): what is below 2^-29 of the largest loses
    // bits, instead of what is below 2^-14.
    static constexpr float UP = std::is_same<Mma, __half>::value ? 15.0f : 0.0f, DOWN = std::is_same<Mma, __half>::value ? 0x1p-15f : 1.0f;
    // What x' has besides log2 s, such that the sums of 8-bit caches are 2^12 times as large as they need be.
    static constexpr float BESIDE = NARROW ? UP - 12.0f : 0.0f;
    static constexpr int STEPS = DP / 16;                   // of the first product
    static constexpr int HALVES = DP / 64;                  // of the second, 64 dimensions each
    static constexpr int PITCH = DP + 4;                    // of a row of partial results in shared memory, in floats
    static_assert(16 * PITCH * 4 + 256 <= STAGES * STAGE, "a warp's partial result takes the place of its ring");

    // Where piece c of vector r lies in a tile.  Eight lanes read 128 bytes at a time: four pieces of two neighbouring keys, one
    // or two of four values two rows apart; the pieces are swapped about so that those lie in different banks.
    static __device__ __forceinline__ int key_at(int r, int c) {
        const int g = r * CHUNKS + c;
        return CHUNKS >= 8 ? (g ^ ((r & 1) << 2)) * 16 : g * 16;
    }
    static __device__ __forceinline__ int value_at(int r, int c) { return ((r * CHUNKS + c) ^ (r & 6)) * 16; }
};

// What results are relative to: 2^(origin factor + near), the largest exponent; near is -infinity where there is none.  ORIGINS: they are not
// all 0 (8-bit caches).
struct Frame {
    float origin, factor, near;
    static __device__ __forceinline__ Frame none() { return {0.0f, 0.0f, NEG_INFINITY}; }
    template <bool ORIGINS>
    __device__ __forceinline__ float less(const Frame &f) const { return ORIGINS ? fmaf(origin - f.origin, factor, near - f.near) : near - f.near; }
    __device__ __forceinline__ float exponent() const { return fmaf(origin, factor, near); }
};

// Running results of 8 NT rows in a warp: with n = lane / 4 and j = lane % 4 a lane has rows 8 nt + 2 j + c, c = 0, 1.
template <typename S, int NT>
struct Running {
    static constexpr int HALVES = S::HALVES;
    float m[NT][2], l[NT][2];     // (l: the lane's share until sum_up)
    float origin[NT][2];          // 8 bits: of the scores that m has been taken from
    float o[HALVES][4][NT][4];    // [h][i][nt][2 e + c]: dimension 64 h + 8 n + 2 i + e
    __device__ __forceinline__ void reset() {
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            m[nt][0] = m[nt][1] = NEG_INFINITY;
            l[nt][0] = l[nt][1] = origin[nt][0] = origin[nt][1] = 0.0f;
#pragma unroll
            for (int h = 0; h < HALVES; ++h)
#pragma unroll
                for (int i = 0; i < 4; ++i)
#pragma unroll
                    for (int e = 0; e < 4; ++e) o[h][i][nt][e] = 0.0f;
        }
    }
    __device__ __forceinline__ void sum_up() {
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int c = 0; c < 2; ++c)
#pragma unroll
                for (int d = 4; d < 32; d <<= 1) l[nt][c] += __shfl_xor_sync(0xFFFFFFFFu, l[nt][c], d);
    }
    // A row's frame, its sum, and eight dimensions.  (The sum of a 16-bit cache without the factor 2^UP, of an 8-bit one with its own, and
    // results to go with it.)
    __device__ __forceinline__ Frame frame(int nt, int c, float factor) const {
        return S::NARROW ? Frame{origin[nt][c], factor, m[nt][c] - S::UP} : Frame{0.0f, 0.0f, m[nt][c] * factor};
    }
    __device__ __forceinline__ float sum(int nt, int c) const { return S::NARROW ? l[nt][c] : l[nt][c] * S::DOWN; }
    __device__ __forceinline__ void eight(int h, int nt, int c, float (&y)[8]) const {
        constexpr float BY = S::NARROW ? S::DOWN * 0x1p12f : S::DOWN;
#pragma unroll
        for (int i = 0; i < 8; ++i) y[i] = o[h][i / 2][nt][2 * (i & 1) + c] * BY;
    }
};

// Queries as the second operand of the first product: a lane loads rows 8 nt + n.
template <typename KV, int DP, int NT>
struct Queries {
    using S = Shape<KV, DP>;
    uint32_t b[S::STEPS][NT][2];
    float factor[NT][2];          // of the scores of the lane's result rows, above 0; the sign is in the queries

    static constexpr int PER = S::NARROW ? 2 : 1;      // 16-byte loads that make up a lane's share of a piece of a key
    struct Raw {
        uint4 x[NT][S::CHUNKS / 4][PER];
    };
    // row[nt]: NULL for none
    static __device__ __forceinline__ void ask(Raw &raw, const uint16_t *const (&row)[NT], int head_dim, int j) {
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int kk = 0; kk < S::CHUNKS / 4; ++kk)
#pragma unroll
                for (int half = 0; half < PER; ++half) {
                    const int d = ((kk * 4 + j) * PER + half) * 8;
                    raw.x[nt][kk][half] = row[nt] && d < head_dim ? *reinterpret_cast<const uint4 *>(row[nt] + d) : make_uint4(0, 0, 0, 0);
                }
    }
    __device__ __forceinline__ void take(const Raw &raw, bool bf16, float scale, int j) {
        // (2^-149 for 0: a score that stands for nothing stays -inf, and any other is 0 to 10^-6)
        const float up = fmaxf(fabsf(scale), 0x1p-149f);
        const uint32_t sign = scale < 0.0f ? 0x80008000u : 0u;
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            factor[nt][0] = factor[nt][1] = up;
            uint32_t top = 0;
#pragma unroll
            for (int kk = 0; kk < S::CHUNKS / 4; ++kk)
#pragma unroll
                for (int half = 0; half < PER; ++half) {
                    const uint4 x = raw.x[nt][kk][half];
                    const uint32_t w[4] = {x.x ^ sign, x.y ^ sign, x.z ^ sign, x.w ^ sign};
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        b[(kk * PER + half) * 2 + i / 2][nt][i & 1] = w[i];
                        if constexpr (S::NARROW) {
                            const float2 f = bf16 ? unpack(w[i], __nv_bfloat16{}) : unpack(w[i], __half{});
                            top = max(top, max(__float_as_uint(f.x) & 0x7FFFFFFFu, __float_as_uint(f.y) & 0x7FFFFFFFu));
                        }
                    }
                }
            if constexpr (S::NARROW) {
                top = max(top, __shfl_xor_sync(0xFFFFFFFFu, top, 1));
                top = max(top, __shfl_xor_sync(0xFFFFFFFFu, top, 2));
                const uint32_t e = min(max(top >> 23, 1u), 253u);
                const float down = __uint_as_float((254u - e) << 23);
#pragma unroll
                for (int st = 0; st < S::STEPS; ++st)
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        uint32_t &w = b[st][nt][i];
                        const float2 f = bf16 ? unpack(w, __nv_bfloat16{}) : unpack(w, __half{});
                        w = pack<__half>(f.x * down, f.y * down);
                    }
#pragma unroll
                for (int c = 0; c < 2; ++c)
                    factor[nt][c] = fminf(fmaxf(up * __uint_as_float(__shfl_sync(0xFFFFFFFFu, e, (2 * j + c) * 4) << 23), 0x1p-149f), 0x1.FFFFFEp127f);
            }
        }
    }
};

// Vectors of zeros with the scale 1 among a tile's values: bit 2 s + e for position 16 s + n + 8 e.
template <typename KV, int DP>
__device__ __forceinline__ uint32_t zeros_of_scale_1(uint32_t values, const float *scales) {
    using S = Shape<KV, DP>;
    const int lane = threadIdx.x & 31, n = lane >> 2, j = lane & 3;
    uint32_t ones = 0, some = 0;
#pragma unroll
    for (int i = 0; i < 2 * S::SUBS; ++i) {
        const int r = n + 8 * i;
        if (scales[S::TILE + r] == 1.0f) ones |= 1u << i;
        uint32_t x = 0;
#pragma unroll
        for (int kk = 0; kk < S::CHUNKS / 4; ++kk) {
            const uint4 v = load16(values + S::value_at(r, kk * 4 + j));
            x |= v.x | v.y | v.z | v.w;
        }
        if (x & (std::is_same<KV, E4m3>::value ? 0x7F7F7F7Fu : 0xFFFFFFFFu)) some |= 1u << i;      // (-0 is 0)
    }
    some |= __shfl_xor_sync(0xFFFFFFFFu, some, 1);
    some |= __shfl_xor_sync(0xFFFFFFFFu, some, 2);
    return ones & ~some;
}

// A tile: keys at `keys`, values at `values` in shared memory; bit i of `real`: position i counts.  scales: TILE of keys,
// then TILE of values.  ENDS: a row takes in the positions before its end only (in the tile); values have to be finite, for
// those behind it get the weight 0.  PART: the positions that do not count may hold anything (otherwise zeros), and only rows whose
// end is not 0 take them in; whatever the positions hold, the other rows stay as they are.
//
// 8 bits: a tile with a value's scale that is not usual, one where a vector of zeros might raise the maximum, and one for which an
// origin has to move, are not taken in (false), but left to the CAREFUL form.  That one moves origins and does not take the tile in
// either, up to twice (`moves`: how often so far).
enum Rows { ALL_ROWS, ENDS, PART_OF_ROWS };
template <typename KV, int DP, int NT, Rows ROWS, bool CAREFUL>
__device__ __forceinline__ bool take_tile(Running<Shape<KV, DP>, NT> &run, const Queries<KV, DP, NT> &q, uint32_t keys, uint32_t values,
                                          const float *scales, uint32_t real, int n, int j, const int (&ends)[NT][2], int moves = 0) {
    using S = Shape<KV, DP>;
    constexpr bool PART = ROWS == PART_OF_ROWS;
    using Mma = typename S::Mma;
    constexpr float LEAST = 0x1p-96f;
    float up[S::SUBS][2];                    // log2 of a value's scale, and BESIDE
    bool odd = false;                        // some scales are below LEAST, infinite or NaN
    float x[S::SUBS][NT][4] = {};            // [2 e + c]: of position 16 s + n + 8 e
#pragma unroll
    for (int kk = 0; kk < S::CHUNKS / 4; ++kk)
#pragma unroll
        for (int s = 0; s < S::SUBS; ++s) {
            const uint4 k0 = load16(keys + S::key_at(s * 16 + n, kk * 4 + j)), k1 = load16(keys + S::key_at(s * 16 + n + 8, kk * 4 + j));
            const uint32_t w0[4] = {k0.x, k0.y, k0.z, k0.w}, w1[4] = {k1.x, k1.y, k1.z, k1.w};
            if constexpr (!S::NARROW) {
#pragma unroll
                for (int st = 0; st < 2; ++st) {
                    const uint32_t a[4] = {w0[2 * st], w1[2 * st], w0[2 * st + 1], w1[2 * st + 1]};
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt) multiply(x[s][nt], a, q.b[2 * kk + st][nt][0], q.b[2 * kk + st][nt][1], Mma{});
                }
            } else {
#pragma unroll
                for (int st = 0; st < 4; ++st) {
                    const uint32_t a[4] = {codes_to_half2(w0[st], 0, KV{}), codes_to_half2(w1[st], 0, KV{}), codes_to_half2(w0[st], 1, KV{}),
                                           codes_to_half2(w1[st], 1, KV{})};
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt) multiply(x[s][nt], a, q.b[4 * kk + st][nt][0], q.b[4 * kk + st][nt][1], Mma{});
                }
            }
        }
    if constexpr (S::NARROW) {
#pragma unroll
        for (int s = 0; s < S::SUBS; ++s)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const float vs = scales[S::TILE + s * 16 + n + 8 * e];
                const bool usual = vs >= LEAST && vs < -NEG_INFINITY;
                up[s][e] = __log2f(!CAREFUL || usual ? vs : LEAST) + S::BESIDE;
                odd |= CAREFUL ? !usual : !(fabsf(up[s][e] - (S::BESIDE + 16.0f)) < 112.0f);      // (the border of 2^-96 is below all that is written)
            }
    }
    if constexpr (S::NARROW) {
#pragma unroll
        for (int s = 0; s < S::SUBS; ++s)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const float ks = scales[s * 16 + n + 8 * e];
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int c = 0; c < 2; ++c) x[s][nt][2 * e + c] = fmaf(x[s][nt][2 * e + c], ks, -run.origin[nt][c]);
            }
    }
    if (PART || real != S::ALL) {
#pragma unroll
        for (int s = 0; s < S::SUBS; ++s)
#pragma unroll
            for (int e = 0; e < 2; ++e)
                if (!((real >> (s * 16 + n + 8 * e)) & 1u)) {
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt) x[s][nt][2 * e] = x[s][nt][2 * e + 1] = NEG_INFINITY;
                }
    }
    if constexpr (PART) {
#pragma unroll
        for (int s = 0; s < S::SUBS; ++s)
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    if (ends[nt][i & 1] == 0) x[s][nt][i] = NEG_INFINITY;
    }
    if constexpr (ROWS == ENDS) {
#pragma unroll
        for (int s = 0; s < S::SUBS; ++s)
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    if (s * 16 + n + 8 * (i >> 1) >= ends[nt][i & 1]) x[s][nt][i] = NEG_INFINITY;
    }
    // maxima: of x itself, which the factor (above 0) multiplies later; with scales of x' = factor x + up
    if constexpr (S::NARROW) {
#pragma unroll
        for (int s = 0; s < S::SUBS; ++s)
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int i = 0; i < 4; ++i) x[s][nt][i] = fmaf(x[s][nt][i], q.factor[nt][i & 1], up[s][i >> 1]);
    }
    float base[NT][2], shrink[NT][2];
    bool grew = false;
    const auto maxima = [&] {
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int c = 0; c < 2; ++c) {
                float m = run.m[nt][c];
#pragma unroll
                for (int s = 0; s < S::SUBS; ++s)
#pragma unroll
                    for (int e = 0; e < 2; ++e) m = fmaxf(m, x[s][nt][2 * e + c]);
#pragma unroll
                for (int d = 4; d < 32; d <<= 1) m = fmaxf(m, __shfl_xor_sync(0xFFFFFFFFu, m, d));
                base[nt][c] = m;
                grew |= m > run.m[nt][c] || (S::NARROW && run.l[nt][c] > 0x1p112f);
            }
    };
    maxima();
    if (__any_sync(0xFFFFFFFFu, grew || (!CAREFUL && odd))) {
        bool zeros = false;                  // with the scale 1
        if constexpr (S::NARROW) {
            bool ones = false;
#pragma unroll
            for (int s = 0; s < S::SUBS; ++s) ones |= up[s][0] == S::BESIDE || up[s][1] == S::BESIDE;
            if (__any_sync(0xFFFFFFFFu, ones)) {
                const uint32_t which = zeros_of_scale_1<KV, DP>(values, scales);
                zeros = which != 0;
                if constexpr (CAREFUL) {
#pragma unroll
                    for (int s = 0; s < S::SUBS; ++s)
#pragma unroll
                        for (int e = 0; e < 2; ++e)
                            if ((which >> (2 * s + e)) & 1u) {
                                up[s][e] -= 96.0f;
#pragma unroll
                                for (int nt = 0; nt < NT; ++nt) x[s][nt][2 * e] -= 96.0f, x[s][nt][2 * e + 1] -= 96.0f;
                            }
                }
            }
        }
        if constexpr (S::NARROW && !CAREFUL) {
            odd = false;                     // (positions that do not count have no scale either)
#pragma unroll
            for (int s = 0; s < S::SUBS; ++s)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const int at = s * 16 + n + 8 * e;
                    const float vs = scales[S::TILE + at];
                    if (!((real >> at) & 1u))
                        up[s][e] = S::BESIDE;
                    else
                        odd |= !(vs > LEAST && vs < -NEG_INFINITY);
                }
        }
        if (CAREFUL && __any_sync(0xFFFFFFFFu, zeros)) maxima();
        bool far = false;
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int c = 0; c < 2; ++c) far |= S::NARROW && base[nt][c] > run.m[nt][c] && fabsf(base[nt][c]) > 256.0f;
        if (S::NARROW && !CAREFUL && __any_sync(0xFFFFFFFFu, zeros || odd || far)) return false;
        // x' of a few hundred has more bits behind the point than a weight: where there is more the origin follows.  (The second time
        // takes what the first one's rounding left.)
        if (CAREFUL && moves < 2 && __any_sync(0xFFFFFFFFu, far)) {
            bool moved = false;
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int c = 0; c < 2; ++c) {
                    const float was = run.origin[nt][c], to = was + base[nt][c] / q.factor[nt][c], by = to - was;
                    if (base[nt][c] > run.m[nt][c] && fabsf(base[nt][c]) > 256.0f && fabsf(to) < -NEG_INFINITY && fabsf(by) < -NEG_INFINITY && by != 0.0f) {
                        run.origin[nt][c] = to;
                        run.m[nt][c] -= by * q.factor[nt][c];
                        moved = true;
                    }
                }
            if (__any_sync(0xFFFFFFFFu, moved)) return false;
        }
        // (lanes of a row have shares of their own, but one maximum)
        if constexpr (S::NARROW) {
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int c = 0; c < 2; ++c) {
                    float l = run.l[nt][c];
#pragma unroll
                    for (int d = 4; d < 32; d <<= 1) l = fmaxf(l, __shfl_xor_sync(0xFFFFFFFFu, l, d));
                    if (l > 0x1p112f) base[nt][c] += 8.0f;
                }
        }
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
            for (int c = 0; c < 2; ++c) {
                const float less = (run.m[nt][c] - base[nt][c]) * (S::NARROW ? 1.0f : q.factor[nt][c]);
                const bool more = base[nt][c] > run.m[nt][c];
                shrink[nt][c] = more ? power2(less) : 1.0f;
                run.m[nt][c] = base[nt][c];
                // (by halves: scales may differ by more than 2^126)
                if constexpr (S::NARROW) {
                    const float half = more ? power2(0.5f * less) : 1.0f;
                    run.l[nt][c] = run.l[nt][c] * half * half;
                } else {
                    run.l[nt][c] *= shrink[nt][c];
                }
            }
#pragma unroll
            for (int h = 0; h < S::HALVES; ++h)
#pragma unroll
                for (int i = 0; i < 4; ++i)
#pragma unroll
                    for (int e = 0; e < 4; ++e) run.o[h][i][nt][e] *= shrink[nt][e & 1];
        }
    }
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int c = 0; c < 2; ++c) {
            const float m = run.m[nt][c];
            base[nt][c] = m == NEG_INFINITY ? 0.0f : S::NARROW ? m - S::UP : m;
        }
    // Weights go into the second product in its type: off by half a step of it (bf16 2^-8, fp16 2^-11; fp32 ones would take two products
    // each), which the many positions that make up a row mostly even out.  The sum takes them as they were, so that it is exact to fp32.
    uint32_t p[S::SUBS][NT][2];
    const auto weigh = [&](auto some_odd) {
        constexpr bool ODD = decltype(some_odd)::value;
#pragma unroll
        for (int s = 0; s < S::SUBS; ++s)
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const int at = s * 16 + n + 8 * e;
                    const float vs = ODD ? scales[S::TILE + at] : 0.0f;
                    float y[2];
#pragma unroll
                    for (int c = 0; c < 2; ++c) {
                        const float z = x[s][nt][2 * e + c] - base[nt][c];
                        y[c] = power2(S::NARROW ? z : fmaf(z, q.factor[nt][c], S::UP));
                        const float weight = S::NARROW ? power2(z - up[s][e]) : y[c];
                        run.l[nt][c] += weight;
                        if (ODD && vs < LEAST)
                            y[c] *= vs * (1.0f / LEAST);
                        else if (ODD && !(vs < -NEG_INFINITY) && (!PART || ((real >> at) & 1u)))
                            y[c] = weight == 0.0f ? __uint_as_float(0x7FC00000u) : vs;
                    }
                    p[s][nt][e] = transpose8x8(pack<Mma>(y[0], y[1]));
                }
    };
    if (CAREFUL && __any_sync(0xFFFFFFFFu, odd))
        weigh(std::true_type{});
    else
        weigh(std::false_type{});
    const auto add = [&](float (&o)[NT][4], int s, uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3) {
        const uint32_t v[4] = {a0, a1, a2, a3};
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            if constexpr (PART) {
                float y[4] = {};
                multiply(y, v, p[s][nt][0], p[s][nt][1], Mma{});
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    if (ends[nt][i & 1] != 0) o[nt][i] += y[i];
            } else {
                multiply(o[nt], v, p[s][nt][0], p[s][nt][1], Mma{});
            }
        }
    };
#pragma unroll
    for (int s = 0; s < S::SUBS; ++s)
#pragma unroll
        for (int h = 0; h < S::HALVES; ++h) {
            const int r[4] = {s * 16 + 2 * j, s * 16 + 2 * j + 1, s * 16 + 2 * j + 8, s * 16 + 2 * j + 9};
            if constexpr (!S::NARROW) {
                uint4 v[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    v[i] = load16(values + S::value_at(r[i], h * 8 + n));
                    if (PART && !((real >> r[i]) & 1u)) v[i] = make_uint4(0, 0, 0, 0);
                }
                const uint32_t w[4][4] = {{v[0].x, v[0].y, v[0].z, v[0].w}, {v[1].x, v[1].y, v[1].z, v[1].w},
                                          {v[2].x, v[2].y, v[2].z, v[2].w}, {v[3].x, v[3].y, v[3].z, v[3].w}};
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    add(run.o[h][i], s, __byte_perm(w[0][i], w[1][i], 0x5410), __byte_perm(w[0][i], w[1][i], 0x7632),
                        __byte_perm(w[2][i], w[3][i], 0x5410), __byte_perm(w[2][i], w[3][i], 0x7632));
            } else {
                uint2 v[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    v[i] = load8(values + S::value_at(r[i], h * 4 + n / 2) + (n & 1) * 8);
                    if (PART && !((real >> r[i]) & 1u)) v[i] = make_uint2(0, 0);
                }
                const uint32_t w[4][2] = {{v[0].x, v[0].y}, {v[1].x, v[1].y}, {v[2].x, v[2].y}, {v[3].x, v[3].y}};
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const uint32_t sel = i & 1 ? 0x7362 : 0x5140;
                    const uint32_t lo = __byte_perm(w[0][i / 2], w[1][i / 2], sel), hi = __byte_perm(w[2][i / 2], w[3][i / 2], sel);
                    add(run.o[h][i], s, codes_to_half2(lo, 0, KV{}), codes_to_half2(lo, 1, KV{}), codes_to_half2(hi, 0, KV{}), codes_to_half2(hi, 1, KV{}));
                }
            }
        }
    return true;
}

// Called, and what it works on goes through local memory: in the loops it cost them registers and order.  (64 x 16384 int8 327 us instead
// of 299, 32 x 8 beams int8 125 instead of 114, e4m3 106 instead of 94.)
template <typename KV, int DP, int NT>
struct Careful {
    Running<Shape<KV, DP>, NT> run;
    Queries<KV, DP, NT> q;
    int ends[NT][2];
};
template <typename KV, int DP, int NT, Rows ROWS>
__device__ __noinline__ void take_carefully(Careful<KV, DP, NT> &c, uint32_t keys, const float *scales, uint32_t real) {
    using S = Shape<KV, DP>;
    const int lane = threadIdx.x & 31;
    Running<S, NT> run = c.run;
    const Queries<KV, DP, NT> q = c.q;
    int ends[NT][2], moves = 0;
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) ends[nt][0] = c.ends[nt][0], ends[nt][1] = c.ends[nt][1];
#pragma unroll 1
    while (!take_tile<KV, DP, NT, ROWS, true>(run, q, keys, keys + S::PLANE, scales, real, lane >> 2, lane & 3, ends, moves)) ++moves;
    c.run = run;
}

// ---- where things are ------------------------------------------------------------------------------------------

// A run of units with the same rows and head that a block works on as one.
struct Pair {
    int64_t first;            // unit
    int32_t units;
    int32_t group, head, row_block;
    int32_t from, to, seq;    // positions, and a sequence whose table has them
};

// Where results go.
template <int DP>
struct Results {
    static constexpr int PART_ROW = DP + 4;       // floats of a row's partial result: o, its frame, l

    const CacheDev &cache;
    const AttendArgs &a;

    // Scratch for the rows of what began before a block's or worker's share (which = 0) or within it (1): nothing else is left
    // unfinished at its ends.
    __device__ __forceinline__ float *block_part(int block, int which, int row) const {
        return a.block_parts + (((int64_t)block * 2 + which) * PART_ROWS + row) * PART_ROW;
    }
    __device__ __forceinline__ float *warp_part(int worker, int sub, int which, int row) const {
        return a.warp_parts + ((((int64_t)worker * a.together + sub) * 2 + which) * a.part_rows + row) * PART_ROW;
    }
    __device__ __forceinline__ float *kept(float *rows, int t, int q_head) const { return rows + ((int64_t)t * a.n_q_heads + q_head) * PART_ROW; }

    template <int N>
    __device__ __forceinline__ void store_row(int t, int q_head, int d, const Frame &f, float l, const float (&y)[N]) const {
        // (no score, or one beyond fp32's range)
        const bool nothing = f.near == NEG_INFINITY && l == l;
        if (f.exponent() == -NEG_INFINITY) l = __uint_as_float(0x7FC00000u);
        const float by = 1.0f / l;
        uint32_t w[N / 2];
#pragma unroll
        for (int e = 0; e < N; e += 2) {
            const float y0 = nothing ? 0.0f : y[e] * by, y1 = nothing ? 0.0f : y[e + 1] * by;
            w[e / 2] = a.q_bf16 ? pack<__nv_bfloat16>(y0, y1) : pack<__half>(y0, y1);
        }
        uint16_t *to = a.out + t * a.out_stride + (int64_t)q_head * cache.head_dim + d;
        if constexpr (N == 8)
            *reinterpret_cast<uint4 *>(to) = make_uint4(w[0], w[1], w[2], w[3]);
        else if constexpr (N == 4)
            *reinterpret_cast<uint2 *>(to) = make_uint2(w[0], w[1]);
        else
            *reinterpret_cast<uint32_t *>(to) = w[0];
        if (a.lse && d == 0)
            a.lse[(int64_t)t * a.n_q_heads + q_head] = nothing ? NEG_INFINITY : (f.exponent() + log2f(l)) * 0.693147180559945f;
    }
    // (the frame and l lie behind the dimensions)
    __device__ __forceinline__ void keep_row(float *row, int d, const Frame &f, float l, const float (&y)[8]) const {
        *reinterpret_cast<float4 *>(row + d) = make_float4(y[0], y[1], y[2], y[3]);
        *reinterpret_cast<float4 *>(row + d + 4) = make_float4(y[4], y[5], y[6], y[7]);
        if (d == 0) *reinterpret_cast<float4 *>(row + DP) = make_float4(f.origin, f.factor, f.near, l);
    }
    // What a partial result counts beside frame `top`.  (Without a maximum its sum is 0, or NaN, which stays.)
    template <bool ORIGINS>
    static __device__ __forceinline__ float weight(const Frame &f, float l, const Frame &top) {
        return f.near == NEG_INFINITY ? (l == l ? 0.0f : 1.0f) : power2(f.less<ORIGINS>(top));
    }
    // The same for its sum, which may be so large that it counts beside a weight below fp32's range (with origins, that is, scales).
    template <bool ORIGINS>
    static __device__ __forceinline__ float weighed(const Frame &f, float l, const Frame &top, float weight) {
        if (!ORIGINS) return l * weight;
        const float half = f.near == NEG_INFINITY ? (l == l ? 0.0f : 1.0f) : power2(0.5f * f.less<ORIGINS>(top));
        return l * half * half;
    }

    __device__ __forceinline__ int group_of(int t) const { return a.grouped ? t / a.group : t; }

    // What the joining kernel has to know of a pair: its pieces, whether the first begins within its worker's (or block's) share, and
    // that worker (or block).  Written by whoever has the first piece; {0, 0} where there is no such pair, {-1, 0} where the token
    // has no row.
    static __device__ __forceinline__ int2 cut(int pieces, int which, int worker) { return make_int2(pieces * 2 + which, worker); }
    __device__ __forceinline__ int2 &shared_cut(int g, int head, int row_block) const {
        return a.shared_cuts[((int64_t)g * cache.n_heads + head) * a.shared_row_blocks + row_block];
    }
    __device__ __forceinline__ int2 &own_cut(int t, int head, int row_block) const {
        return a.own_cuts[((int64_t)t * cache.n_heads + head) * a.row_blocks + row_block];
    }
};

// WARPS warps per row; those that were not cut are stored already.  A row's partial results are asked for AHEAD at a time and joined
// in a fixed order: by eights, every WARPS-th eight by a warp, and then the warps.  Latencies: 2 to 5 us, of which a launch is one.  (In
// the first kernel, by whichever warp is the last to be done with a token, the same took 6.5 us at the end of all others,
// most of it on an atomic's way and back, and its registers cost the loops theirs.)
template <int DP, int WARPS, bool ORIGINS>
__global__ void __launch_bounds__(ATTEND_THREADS)
attend_join_kernel(const __grid_constant__ CacheDev cache, const __grid_constant__ AttendArgs a) {
    attend_enter();
    using R = Results<DP>;
    constexpr int PER = DP / 32, AHEAD = 8;      // dimensions of a lane
    const R to{cache, a};
    __shared__ float rows[WARPS > 1 ? ATTEND_WARPS : 1][R::PART_ROW];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, which = warp % WARPS;
    const int t = blockIdx.y, q_head = ((int)blockIdx.x * ATTEND_WARPS + warp) / WARPS;
    if (q_head >= a.n_q_heads) return;
    const int g = to.group_of(t), head = q_head / a.rows, r = q_head - head * a.rows, sub = head % a.together;
    int2 x = make_int2(0, 0), z = make_int2(0, 0);
    int x_row = 0, z_row = 0;
    if (a.shared_row_blocks > 0) {
        const int i = (t - g * a.group) * a.rows + r, b = i / a.shared_rows_each;
        x_row = i - b * a.shared_rows_each;
        x = to.shared_cut(g, head, b);
    }
    if (a.grouped || a.shared_row_blocks == 0) {
        const int b = r / a.warp_rows;
        z_row = r - b * a.warp_rows;
        z = to.own_cut(t, head, b);
    }
    if (z.x < 0) return;
    const int n_x = x.x >> 1, n_z = z.x >> 1, n = n_x + n_z;
    if (n <= 1) return;                       // stored already, or there is nothing
    // (what is not a pair's first piece begins with its share)
    const auto piece = [&](int i) -> const float * {
        if (i < n_x) return n_x == 1 ? to.kept(a.shared_rows, t, q_head) : to.block_part(x.y + i, i == 0 ? x.x & 1 : 0, x_row);
        i -= n_x;
        return n_z == 1 ? to.kept(a.own_rows, t, q_head) : to.warp_part(z.y + i, sub, i == 0 ? z.x & 1 : 0, z_row);
    };
    Frame m = Frame::none();
    float l = 0.0f, y[PER] = {};
    for (int i0 = which * AHEAD; i0 < n; i0 += WARPS * AHEAD) {
        const int here = min(AHEAD, n - i0);
        const float *mine = piece(i0 + min(lane % AHEAD, here - 1));
        float4 st = __ldcg(reinterpret_cast<const float4 *>(mine + DP));
        float2 f[AHEAD][PER / 2];
#pragma unroll
        for (int k = 0; k < AHEAD; ++k) {
            const float *p = reinterpret_cast<const float *>(__shfl_sync(0xFFFFFFFFu, (unsigned long long)(uintptr_t)mine, k)) + lane * PER;
#pragma unroll
            for (int e = 0; e < PER / 2; ++e) f[k][e] = __ldcg(reinterpret_cast<const float2 *>(p) + e);
        }
        if (lane % AHEAD >= here) st = make_float4(0.0f, 0.0f, NEG_INFINITY, 0.0f);
        const Frame at{st.x, st.y, st.z};
        Frame top = at;
#pragma unroll
        for (int o = AHEAD / 2; o > 0; o >>= 1) {
            if (!ORIGINS) {
                top.near = fmaxf(top.near, __shfl_xor_sync(0xFFFFFFFFu, top.near, o));
                continue;
            }
            const Frame x{__shfl_xor_sync(0xFFFFFFFFu, top.origin, o), __shfl_xor_sync(0xFFFFFFFFu, top.factor, o), __shfl_xor_sync(0xFFFFFFFFu, top.near, o)};
            if (x.less<ORIGINS>(top) > 0.0f) top = x;
        }
        // (frames that are equal up to rounding may have left lanes with different ones)
        if (ORIGINS) top = {__shfl_sync(0xFFFFFFFFu, top.origin, 0), __shfl_sync(0xFFFFFFFFu, top.factor, 0), __shfl_sync(0xFFFFFFFFu, top.near, 0)};
        if (!ORIGINS)
            top.near = fmaxf(top.near, m.near);
        else if (m.less<ORIGINS>(top) > 0.0f)
            top = m;
        const float w = R::template weight<ORIGINS>(at, st.w, top), old = R::template weight<ORIGINS>(m, l, top);
        float sum = R::template weighed<ORIGINS>(at, st.w, top, w);
#pragma unroll
        for (int o = AHEAD / 2; o > 0; o >>= 1) sum += __shfl_xor_sync(0xFFFFFFFFu, sum, o);
        l = R::template weighed<ORIGINS>(m, l, top, old) + sum;
        m = top;
#pragma unroll
        for (int e = 0; e < PER; ++e) y[e] *= old;
#pragma unroll
        for (int k = 0; k < AHEAD; ++k) {
            const float by = __shfl_sync(0xFFFFFFFFu, w, k);
            if (k < here) {
#pragma unroll
                for (int e = 0; e < PER / 2; ++e) y[2 * e] += f[k][e].x * by, y[2 * e + 1] += f[k][e].y * by;
            }
        }
    }
    if constexpr (WARPS > 1) {                // (a block has one row then, and all of its warps come here)
        static_assert(WARPS == ATTEND_WARPS, "");
#pragma unroll
        for (int e = 0; e < PER; ++e) rows[warp][lane * PER + e] = y[e];
        if (lane == 0) rows[warp][DP] = m.origin, rows[warp][DP + 1] = m.factor, rows[warp][DP + 2] = m.near, rows[warp][DP + 3] = l;
        __syncthreads();
        if (warp > 0) return;
        for (int w = 1; w < min(WARPS, (n + AHEAD - 1) / AHEAD); ++w) {
            const Frame mw{rows[w][DP], rows[w][DP + 1], rows[w][DP + 2]}, top = mw.less<ORIGINS>(m) > 0.0f ? mw : m;
            const float lw = rows[w][DP + 3], old = R::template weight<ORIGINS>(m, l, top), by = R::template weight<ORIGINS>(mw, lw, top);
            l = R::template weighed<ORIGINS>(m, l, top, old) + R::template weighed<ORIGINS>(mw, lw, top, by), m = top;
#pragma unroll
            for (int e = 0; e < PER; ++e) y[e] = y[e] * old + rows[w][lane * PER + e] * by;
        }
    }
    if (lane * PER < cache.head_dim) to.template store_row<PER>(t, q_head, lane * PER, m, l, y);
}

// SHARED_WARPS: so many of a block's warps work on the same tiles, each for 8 NTS rows of its own; 0: there are no pairs for
// whole blocks.  A warp by itself works for 8 NT rows.
template <typename KV, int DP, int SHARED_WARPS, bool GROUPED, int NTS, int NT>
struct Attend : Results<DP> {
    using R = Results<DP>;
    using R::cache, R::a, R::PART_ROW, R::block_part, R::warp_part, R::kept, R::keep_row, R::group_of;
    using S = Shape<KV, DP>;
    static constexpr int WM = SHARED_WARPS == 0 ? 1 : SHARED_WARPS;
    static constexpr int WARP_ROWS = 8 * NT;
    static constexpr int SHARED_ROWS = 8 * NTS;                 // of a warp
    static constexpr int ROWS = SHARED_ROWS * WM;               // of a shared pair
    static constexpr int UNIT = ATTEND_WARPS * S::TILE;         // positions of a shared unit
    // What a pair costs besides its tiles, in units: so many are dealt out in front of its own, and passed over.  (48 ragged sequences
    // of 16 heads, some of a few positions: warps were done after 11 to 22 us without, 14 in the middle.)
    static constexpr int PAIR_COST = 1, SHARED_PAIR_COST = 2;

    Book &book;
    char *ring;
    float *scales;            // [warp][stage][2 TILE]
    uint32_t *real;           // [warp][stage]
    int32_t shared_blocks = 0;      // blocks that work on shared pairs: the first ones

    __device__ Attend(const CacheDev &cache, const AttendArgs &a, Book &book, char *ring, float *scales, uint32_t *real)
        : R{cache, a}, book(book), ring(ring), scales(scales), real(real) {}

    __device__ __forceinline__ int32_t shared_units(int g) const {
        return SHARED_WARPS == 0 ? 0 : tiles_of(GROUPED ? 0 : book.from[g], book.to[g], UNIT);
    }
    __device__ __forceinline__ int32_t own_units(int t) const { return GROUPED || SHARED_WARPS == 0 ? tiles_of(book.from[t], book.end[t], S::TILE) : 0; }

    // ---- tiles ----
    // A warp's tile: lane i knows the block of position `pos` of the tile (i % TILE).  Commits a group of copies.
    __device__ __forceinline__ void copy_tile(int warp, int stage, bool live, int32_t block, uint32_t pos, int head, int lane) const {
        uint32_t slot = 0xFFFFFFFFu;
        if ((uint32_t)block < (uint32_t)cache.n_blocks)
            slot = (uint32_t)block * cache.block.d + (pos - cache.block.quotient(pos) * cache.block.d);
        const uint32_t ok = __ballot_sync(0xFFFFFFFFu, slot != 0xFFFFFFFFu) & S::ALL;
        if (live) {
            constexpr int AT_ONCE = 32 / S::CHUNKS;      // vectors that 32 lanes copy
            const uint32_t width = (uint32_t)cache.head_dim * S::BYTES, step = width * (uint32_t)cache.n_heads;
            const uint32_t keys = shared_address(ring + (warp * S::STAGES + stage) * S::STAGE), values = keys + S::PLANE;
            const int c = lane % S::CHUNKS, r0 = lane / S::CHUNKS;
            const uint64_t offset = (uint64_t)head * width + (uint32_t)c * 16;
            const char *k = cache.k + offset, *v = cache.v + offset;
            if (ok == S::ALL && width == S::CHUNKS * 16) {
#pragma unroll
                for (int it = 0; it < S::TILE / AT_ONCE; ++it) {
                    const int r = it * AT_ONCE + r0;
                    const uint64_t off = (uint64_t)__shfl_sync(0xFFFFFFFFu, slot, r) * step;
                    copy16(keys + S::key_at(r, c), k + off);
                    copy16(values + S::value_at(r, c), v + off);
                }
            } else {
#pragma unroll 1
                for (int it = 0; it < S::TILE / AT_ONCE; ++it) {
                    const int r = it * AT_ONCE + r0;
                    const uint32_t of = __shfl_sync(0xFFFFFFFFu, slot, r);
                    const bool is = ((ok >> r) & 1u) && (uint32_t)c * 16 < width;
                    const uint64_t off = (uint64_t)of * step;
                    copy16(keys + S::key_at(r, c), is ? k + off : cache.k, is);
                    copy16(values + S::value_at(r, c), is ? v + off : cache.v, is);
                }
            }
            if constexpr (S::NARROW) {
                const bool is = slot != 0xFFFFFFFFu;
                const uint64_t at = is ? (uint64_t)slot * (uint32_t)cache.n_heads + head : 0;
                const uint32_t to = shared_address(scales + (warp * S::STAGES + stage) * (2 * S::TILE) + lane % S::TILE);
                if (S::TILE == 32 || lane < 16) copy4(to, cache.k_scale + at, is);
                if (S::TILE == 32 || lane >= 16) copy4(to + S::TILE * 4, cache.v_scale + at, is);
            }
            if (lane == 0) real[warp * S::STAGES + stage] = ok;
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
    }
    // Anything but a block where there is none.  (The last tile of a sequence of nearly 2^31 positions passes that: positions are unsigned.)
    __device__ __forceinline__ int32_t entry(const int32_t *row, uint32_t pos, int to) const {
        return pos < (uint32_t)to ? row[cache.block.quotient(pos)] : -1;
    }
    static __device__ __forceinline__ void wait_tile() { asm volatile("cp.async.wait_group %0;" ::"n"(S::STAGES - 2) : "memory"); }

    // ---- pairs of whole blocks ----
    // The token and query head of row i of a pair (token -1: none).
    __device__ __forceinline__ int row_of(const Pair &p, int i, int &head) const {
        const int r = p.row_block * ROWS + i, m = r / a.rows, t = p.group * a.group + m;
        head = p.head * a.rows + (r - m * a.rows);
        return m < a.group && t < a.n_tokens && book.end[t] > 0 ? t : -1;
    }
    static __device__ __forceinline__ void stream_sync(int stream) {     // the warps that work on the same tiles
        if constexpr (WM == 1)
            __syncwarp();
        else if constexpr (WM == ATTEND_WARPS)
            __syncthreads();
        else
            asm volatile("bar.sync %0, %1;" ::"r"(1 + stream), "n"(32 * WM) : "memory");
    }

    // Whether a tile's values are all finite.
    static __device__ __forceinline__ bool values_finite(uint32_t values, const float *value_scales, int lane) {
        bool odd = false;
        if constexpr (S::NARROW) odd = lane < S::TILE && !(value_scales[lane] < __uint_as_float(0x7F800000u));
        if constexpr (!std::is_same<KV, Int8>::value) {
#pragma unroll 4
            for (int i = lane; i < S::PLANE / 16; i += 32) {
                const uint4 x = load16(values + i * 16);
                const uint32_t w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    if constexpr (S::NARROW)           // (the only one: all bits but the sign set)
                        odd |= (((w[k] & 0x7F7F7F7Fu) + 0x01010101u) & 0x80808080u) != 0;
                    else {
                        constexpr uint32_t top = std::is_same<KV, __half>::value ? 0x7C00u : 0x7F80u;
                        odd |= (w[k] & top) == top || ((w[k] >> 16) & top) == top;
                    }
                }
            }
        }
        return !__any_sync(0xFFFFFFFFu, odd);
    }

    // A tile, whatever is in it.
    template <int ROWS_BY_8, Rows ROWS>
    static __device__ __forceinline__ void take(Running<S, ROWS_BY_8> &run, Queries<KV, DP, ROWS_BY_8> &q, uint32_t keys, const float *scales, uint32_t real,
                                                int n, int j, const int (&ends)[ROWS_BY_8][2]) {
        if constexpr (!S::NARROW) {
            take_tile<KV, DP, ROWS_BY_8, ROWS, false>(run, q, keys, keys + S::PLANE, scales, real, n, j, ends);
        } else {
            if (ROWS != PART_OF_ROWS)
                if (take_tile<KV, DP, ROWS_BY_8, ROWS, false>(run, q, keys, keys + S::PLANE, scales, real, n, j, ends)) return;
            Careful<KV, DP, ROWS_BY_8> c;
            c.run = run, c.q = q;
#pragma unroll
            for (int nt = 0; nt < ROWS_BY_8; ++nt) c.ends[nt][0] = ends[nt][0], c.ends[nt][1] = ends[nt][1];
            take_carefully<KV, DP, ROWS_BY_8, ROWS>(c, keys, scales, real);
            run = c.run, q = c.q;
        }
    }

    // Units [u0, u1) of a pair.  Rows that nothing else belongs to are stored, others kept as partial results.
    __device__ __forceinline__ void segment(const Pair &pair, int64_t u0, int64_t u1) const {
        constexpr int STREAMS = ATTEND_WARPS / WM, STREAM = S::TILE * WM;
        const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, n = lane >> 2, j = lane & 3;
        const int stream = warp / WM, wm = warp % WM;
        const int from = pair.from + (int)(u0 - pair.first) * UNIT;
        const int to = (int)min((int64_t)pair.to, (int64_t)pair.from + (u1 - pair.first) * UNIT);
        const int tiles = tiles_of(from, to, STREAM);                                // of all streams
        const int mine = tiles > stream ? (tiles - stream + STREAMS - 1) / STREAMS : 0;
        const int32_t *row = a.table + pair.seq * a.stride;
        const auto position = [&](int i) { return (uint32_t)from + (uint32_t)(i * STREAMS + stream) * STREAM + (uint32_t)(wm * S::TILE + lane % S::TILE); };
        const auto block_at = [&](int i) { return i < mine ? entry(row, position(i), to) : -1; };
        int32_t first_blocks[S::STAGES - 1];
#pragma unroll
        for (int i = 0; i < S::STAGES - 1; ++i) first_blocks[i] = block_at(i);
        int32_t next = block_at(S::STAGES - 1);
        Queries<KV, DP, NTS> q;
        int ends[NTS][2], least = 0x7FFFFFFF;    // where the lane's rows end; the first of the warp's rows to end
        {
            const uint16_t *rows[NTS];
#pragma unroll
            for (int nt = 0; nt < NTS; ++nt) {
                int head;
                const int t = row_of(pair, wm * SHARED_ROWS + nt * 8 + n, head);
                rows[nt] = t < 0 ? nullptr : a.q + t * a.q_stride + (int64_t)head * cache.head_dim;
                if (GROUPED && t >= 0) least = min(least, book.end[t]);
                if constexpr (GROUPED) {
#pragma unroll
                    for (int c = 0; c < 2; ++c) {
                        const int of = row_of(pair, wm * SHARED_ROWS + nt * 8 + 2 * j + c, head);
                        ends[nt][c] = of < 0 ? 0 : book.end[of];
                    }
                }
            }
            typename Queries<KV, DP, NTS>::Raw raw;
            q.ask(raw, rows, cache.head_dim, j);
#pragma unroll
            for (int i = 0; i < S::STAGES - 1; ++i) copy_tile(warp, i, i < mine, first_blocks[i], position(i), pair.head, lane);
            q.take(raw, a.q_bf16, a.scale, j);
            if constexpr (GROUPED) {
#pragma unroll
                for (int o = 16; o > 0; o >>= 1) least = min(least, __shfl_xor_sync(0xFFFFFFFFu, least, o));
            }
        }
        int in[NTS][2] = {};                    // where the rows end in the tile
        Running<S, NTS> run;
        run.reset();
#pragma unroll 1
        for (int i = 0; i < mine; ++i) {
            wait_tile();
            stream_sync(stream);
            // (the tile that was used last is free: all warps of the stream are past it)
            copy_tile(warp, (i + S::STAGES - 1) % S::STAGES, i + S::STAGES - 1 < mine, next, position(i + S::STAGES - 1), pair.head, lane);
            next = block_at(i + S::STAGES);
            const int stage = i % S::STAGES;
#pragma unroll 1
            for (int w = 0; w < WM; ++w) {
                const int of = (stream * WM + w) * S::STAGES + stage;
                const uint32_t ok = real[of];
                if (!ok) continue;
                const uint32_t keys = shared_address(ring + of * S::STAGE);
                const int at = from + (i * STREAMS + stream) * STREAM + w * S::TILE;
                const float *const its_scales = scales + of * (2 * S::TILE);
                const bool whole = !GROUPED || least - at >= S::TILE;
                if (whole) {
                    take<NTS, ALL_ROWS>(run, q, keys, its_scales, ok, n, j, in);
                    continue;
                }
                // rows that end within the tile, or before it
                if (values_finite(keys + S::PLANE, its_scales + S::TILE, lane)) {
#pragma unroll
                    for (int nt = 0; nt < NTS; ++nt)
#pragma unroll
                        for (int c = 0; c < 2; ++c) in[nt][c] = ends[nt][c] - at;
                    take<NTS, ENDS>(run, q, keys, its_scales, ok, n, j, in);
                    continue;
                }
                // (an infinity or a NaN would reach them with the weight 0: the rows go by themselves)
                int past = 0;
#pragma unroll 1
                while (true) {
                    int e = S::TILE + 1;
#pragma unroll
                    for (int nt = 0; nt < NTS; ++nt)
#pragma unroll
                        for (int c = 0; c < 2; ++c)
                            if (min(ends[nt][c] - at, S::TILE) > past) e = min(e, min(ends[nt][c] - at, S::TILE));
#pragma unroll
                    for (int o = 16; o > 0; o >>= 1) e = min(e, __shfl_xor_sync(0xFFFFFFFFu, e, o));
                    if (e > S::TILE) break;
#pragma unroll
                    for (int nt = 0; nt < NTS; ++nt)
#pragma unroll
                        for (int c = 0; c < 2; ++c) in[nt][c] = min(ends[nt][c] - at, S::TILE) == e;
                    take<NTS, PART_OF_ROWS>(run, q, keys, its_scales, ok & ((2u << (e - 1)) - 1u), n, j, in);
                    past = e;
                }
            }
        }
        asm volatile("cp.async.wait_group 0;" ::: "memory");
        run.sum_up();
        stream_sync(stream);
        // every warp's results into its ring
        float *const part = reinterpret_cast<float *>(ring + warp * S::STAGES * S::STAGE);
        float4 *const stats = reinterpret_cast<float4 *>(part + SHARED_ROWS * S::PITCH);
#pragma unroll
        for (int nt = 0; nt < NTS; ++nt)
#pragma unroll
            for (int c = 0; c < 2; ++c) {
                const int r = nt * 8 + 2 * j + c;
                const Frame f = run.frame(nt, c, q.factor[nt][c]);
                if (n == 0) stats[r] = make_float4(f.origin, f.factor, f.near, run.sum(nt, c));
#pragma unroll
                for (int h = 0; h < S::HALVES; ++h) {
                    float y[8];
                    run.eight(h, nt, c, y);
                    float4 *to = reinterpret_cast<float4 *>(part + r * S::PITCH + h * 64 + n * 8);
                    to[0] = make_float4(y[0], y[1], y[2], y[3]), to[1] = make_float4(y[4], y[5], y[6], y[7]);
                }
            }
        __syncthreads();
        // joined over the streams: a thread takes eight dimensions of a row
        const bool whole = u0 == pair.first && u1 == pair.first + pair.units;
        const int which = book.shared.begin(blockIdx.x) >= pair.first ? 0 : 1;
        if (threadIdx.x == 0 && u0 == pair.first)
            this->shared_cut(pair.group, pair.head, pair.row_block) =
                R::cut(whole ? 1 : book.shared.owner(pair.first + pair.units - 1) - (int)blockIdx.x + 1, which, blockIdx.x);
        const int n_rows = min(ROWS, a.group * a.rows - pair.row_block * ROWS);
        for (int i = threadIdx.x; i < n_rows * (DP / 8); i += ATTEND_THREADS) {
            const int r = i / (DP / 8), d = (i % (DP / 8)) * 8, in_warp = r % SHARED_ROWS;
            const char *base = ring + (r / SHARED_ROWS) * S::STAGES * S::STAGE;
            Frame m = Frame::none();
            float l = 0.0f, y[8] = {};
            float4 st[STREAMS];
#pragma unroll
            for (int s = 0; s < STREAMS; ++s) {
                const float *of = reinterpret_cast<const float *>(base + s * WM * S::STAGES * S::STAGE);
                st[s] = reinterpret_cast<const float4 *>(of + SHARED_ROWS * S::PITCH)[in_warp];
                const Frame f{st[s].x, st[s].y, st[s].z};
                if (f.less<S::NARROW>(m) > 0.0f) m = f;
            }
#pragma unroll
            for (int s = 0; s < STREAMS; ++s) {
                const float *of = reinterpret_cast<const float *>(base + s * WM * S::STAGES * S::STAGE) + in_warp * S::PITCH + d;
                const Frame f{st[s].x, st[s].y, st[s].z};
                const float w = R::template weight<S::NARROW>(f, st[s].w, m);
                l += R::template weighed<S::NARROW>(f, st[s].w, m, w);
#pragma unroll
                for (int e = 0; e < 8; ++e) y[e] += of[e] * w;
            }
            int head;
            const int t = row_of(pair, r, head);
            if (t < 0) continue;
            if (!whole)
                keep_row(block_part(blockIdx.x, which, r), d, m, l, y);
            else if (own_units(t) > 0)
                keep_row(kept(a.shared_rows, t, head), d, m, l, y);
            else if (d < cache.head_dim)
                this->template store_row<8>(t, head, d, m, l, y);
        }
        __syncthreads();      // the rings are free again
    }

    __device__ __forceinline__ void work_on_pairs() const {
        if ((int)blockIdx.x >= book.shared.workers) return;
        int64_t u = book.shared.begin(blockIdx.x);
        const int64_t end = book.shared.begin(blockIdx.x + 1);
        int g = find(book.shared_upto, a.n_groups, u);
#pragma unroll 1
        while (u < end) {
            while (book.shared_upto[g + 1] <= u) ++g;
            Pair p;
            p.units = shared_units(g);
            const int32_t dealt = p.units + SHARED_PAIR_COST;
            const int i = (int)quotient(u - book.shared_upto[g], dealt);
            p.first = book.shared_upto[g] + (int64_t)i * dealt + SHARED_PAIR_COST;
            u = max(u, p.first);
            if (u >= end) break;
            p.group = g;
            p.head = i / a.shared_row_blocks, p.row_block = i % a.shared_row_blocks;
            p.from = GROUPED ? 0 : book.from[g], p.to = book.to[g];
            // (the token that goes furthest has all of the shared positions in its table)
            int t = g * a.group;
            if constexpr (GROUPED)
                for (int m = 1; m < a.group && g * a.group + m < a.n_tokens; ++m)
                    if (book.end[g * a.group + m] > book.end[t]) t = g * a.group + m;
            p.seq = book.seq[t];
            const int64_t stop = min(end, p.first + p.units);
            segment(p, u, stop);
            u = stop;
        }
    }

    // The last i < n with upto[i] <= u.
    static __device__ __forceinline__ int find(const int64_t *upto, int n, int64_t u) {
        int lo = 0, hi = n;
        while (hi - lo > 1) {
            const int mid = (lo + hi) >> 1;
            if (upto[mid] <= u) lo = mid; else hi = mid;
        }
        return lo;
    }

    // ---- pairs of single warps ----
    // A warp's place in its share: tile i of n of a token and one of its runs (key heads by row blocks).
    struct Place {
        int t, run, i, n, from, end;
        const int32_t *row;
    };
    __device__ __forceinline__ void enter(Place &p) const {      // token p.t
        p.from = book.from[p.t], p.end = book.end[p.t];
        p.n = own_units(p.t);
        p.row = a.table + book.seq[p.t] * a.stride;
    }
    __device__ __forceinline__ Place place(int64_t &u) const {   // (u moves on to a unit with a tile)
        Place p;
        p.t = find(book.upto, a.n_tokens, u);
        while (book.upto[p.t + 1] <= u) ++p.t;
        enter(p);
        const int64_t o = u - book.upto[p.t];
        p.run = (int)quotient(o, p.n + PAIR_COST);
        p.i = (int)(o - (int64_t)p.run * (p.n + PAIR_COST)) - PAIR_COST;
        if (p.i < 0) u -= p.i, p.i = 0;
        return p;
    }
    // `runs`: of a token
    __device__ __forceinline__ void step(Place &p, int64_t &u, int runs) const {
        ++u;
        if (++p.i < p.n) return;
        p.i = 0;
        u += PAIR_COST;
        if (++p.run < runs) return;
        p.run = 0;
        do ++p.t;
        while (p.t < a.n_tokens && book.upto[p.t + 1] == book.upto[p.t]);
        if (p.t < a.n_tokens) enter(p);
    }

    // Every warp by itself: the tiles of its share one after the other, whatever they belong to, with copies always
    // STAGES - 1 tiles ahead.  Warps of a block have neighbouring key heads of the same positions where there are enough heads, so
    // that what they read lies together.
    __device__ __forceinline__ void work_alone() const {
        const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, n = lane >> 2, j = lane & 3;
        const int id = ((int)blockIdx.x - shared_blocks) * ATTEND_WARPS + warp;
        const int worker = id / a.together, sub = id - worker * a.together;
        if (worker >= book.own.workers) return;
        const int64_t begin = book.own.begin(worker), end = book.own.begin(worker + 1);
        const int runs = cache.n_heads / a.together * a.row_blocks;
        const auto head_of = [&](int run) { return (a.row_blocks == 1 ? run : run / a.row_blocks) * a.together + sub; };
        int64_t u = begin;
        Place front = place(u), at = front;
        if (u >= end) return;
        int64_t ahead = u;                     // the unit of `front`
        using Q = Queries<KV, DP, NT>;
        typename Q::Raw raw;                   // of the next pair
        const auto ask = [&](const Place &of) {
            const int head = head_of(of.run), row0 = of.run % a.row_blocks * WARP_ROWS;
            const uint16_t *rows[NT];
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
                const int r = row0 + nt * 8 + n;
                rows[nt] = r < a.rows ? a.q + of.t * a.q_stride + (int64_t)(head * a.rows + r) * cache.head_dim : nullptr;
            }
            Q::ask(raw, rows, cache.head_dim, j);
        };
        ask(at);
        const auto fetch = [&](int32_t &block, uint32_t &p, int &head) -> bool {    // the table's entry of the tile in front
            block = -1;
            if (ahead >= end) return false;
            p = (uint32_t)front.from + (uint32_t)front.i * S::TILE + (uint32_t)lane % S::TILE;
            head = head_of(front.run);
            block = entry(front.row, p, front.end);
            step(front, ahead, runs);
            return true;
        };
        int32_t blocks[S::STAGES];
        uint32_t pos[S::STAGES];
        int heads[S::STAGES];
        bool lives[S::STAGES];
#pragma unroll
        for (int i = 0; i < S::STAGES; ++i) lives[i] = fetch(blocks[i], pos[i], heads[i]);
#pragma unroll
        for (int i = 0; i < S::STAGES - 1; ++i) copy_tile(warp, i, lives[i], blocks[i], pos[i], heads[i], lane);
        int32_t block = blocks[S::STAGES - 1];
        uint32_t p = pos[S::STAGES - 1];
        int p_head = heads[S::STAGES - 1];
        bool live = lives[S::STAGES - 1];
        Q q;
        Running<S, NT> run;
        const int in[NT][2] = {};
        int stage = 0;
        bool fresh = true;
#pragma unroll 1
        while (u < end) {
            if (fresh) {
                q.take(raw, a.q_bf16, a.scale, j);
                run.reset();
                Place next = at;
                next.i = next.n - 1;
                int64_t v = u + next.i - at.i;
                step(next, v, runs);
                if (v < end) ask(next);
            }
            wait_tile();
            __syncwarp();
            copy_tile(warp, stage == 0 ? S::STAGES - 1 : stage - 1, live, block, p, p_head, lane);
            live = fetch(block, p, p_head);
            const int of = warp * S::STAGES + stage;
            const uint32_t ok = real[of], keys = shared_address(ring + of * S::STAGE);
            const float *const its_scales = scales + of * (2 * S::TILE);
            if (ok) take<NT, ALL_ROWS>(run, q, keys, its_scales, ok, n, j, in);
            if (++stage == S::STAGES) stage = 0;
            fresh = at.i == at.n - 1;
            if (fresh || u + 1 >= end) finish(run, q, at, u, begin, end, worker, sub, head_of(at.run), at.run % a.row_blocks * WARP_ROWS, n, j, lane);
            step(at, u, runs);
        }
        asm volatile("cp.async.wait_group 0;" ::: "memory");
    }

    __device__ __forceinline__ void finish(Running<S, NT> &run, const Queries<KV, DP, NT> &q, const Place &at, int64_t u, int64_t begin,
                                           int64_t end, int worker, int sub, int head, int row0, int n, int j, int lane) const {
        const int64_t first = u - at.i;
        const bool whole = first >= begin && first + at.n <= end;
        const bool more = GROUPED && shared_units(group_of(at.t)) > 0;
        const int which = begin >= first ? 0 : 1;
        if (lane == 0 && first >= begin)
            this->own_cut(at.t, head, row0 / WARP_ROWS) = R::cut(whole ? 1 : book.own.owner(first + at.n - 1) - worker + 1, which, worker);
        run.sum_up();
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int c = 0; c < 2; ++c) {
                const int r = row0 + nt * 8 + 2 * j + c, q_head = head * a.rows + r;
                if (r >= a.rows) continue;
                float *to_keep = whole ? kept(a.own_rows, at.t, q_head) : warp_part(worker, sub, which, r - row0);
                const Frame m = run.frame(nt, c, q.factor[nt][c]);
                const float l = run.sum(nt, c);
#pragma unroll
                for (int h = 0; h < S::HALVES; ++h) {
                    const int d = h * 64 + n * 8;
                    float y[8];
                    run.eight(h, nt, c, y);
                    if (!whole || more)
                        keep_row(to_keep, d, m, l, y);
                    else if (d < cache.head_dim)
                        this->template store_row<8>(at.t, q_head, d, m, l, y);
                }
            }
    }
};

// Prefix sums of one number a thread over the block, for as many rounds as it takes: `before` everything so far.
__device__ __forceinline__ int64_t sums_before(int64_t n, int64_t &total, int64_t *scan) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    int64_t x = n;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int64_t y = __shfl_up_sync(0xFFFFFFFFu, x, o);
        if (lane >= o) x += y;
    }
    if (lane == 31) scan[warp] = x;
    __syncthreads();
    int64_t before = total;
#pragma unroll
    for (int w = 0; w < ATTEND_WARPS; ++w) {
        if (w < warp) before += scan[w];
        total += scan[w];
    }
    __syncthreads();
    return before + x - n;
}

// What it measured (with the join behind it; from memory, 32 query and 8 key heads of 128): 32 tokens of 4096 positions, bf16: 75 us,
// 5.9 TB/s, 0.90 of a copy's rate, of which the start to the first tile takes 6 us and the end 6; 64 of 16384, e4m3: 284 to 297 us,
// 6.1 to 6.4 TB/s (in long runs, at a lower clock, 305 to 330); one of 1000: 8.5 us; 32 x 8 beams of 1800 that share their prompts: 83 to 87 us, 3.4 TB/s.  The tensor pipe is
// busy for 9 to 18 % of the time, and issue slots are taken to a quarter (16 bits) and to a half (8 bits: 680 instructions a tile).
// Two blocks of four warps on an SM: 210 to 255 registers, three stages of 8 KB a warp.  With head sizes above 128 one block, and
// registers do not suffice for groups, nor for more than 8 rows of a key head: 216 to 1824 bytes of a thread are spilled and loaded.  Three blocks of 168 registers with two
// stages: 492 us instead of 283; tiles of 16 positions in 8-bit caches: 369.
template <typename KV, int DP, int SHARED_WARPS, bool GROUPED, int NTS, int NT>
__global__ void __launch_bounds__(ATTEND_THREADS, Shape<KV, DP>::BLOCKS)
attend_kernel(const __grid_constant__ CacheDev cache, const __grid_constant__ AttendArgs a) {
    using S = Shape<KV, DP>;
    using A = Attend<KV, DP, SHARED_WARPS, GROUPED, NTS, NT>;
    extern __shared__ __align__(128) char ring[];
    __shared__ Book book;
    __shared__ int64_t scan[ATTEND_WARPS];
    __shared__ float scales[S::NARROW ? ATTEND_WARPS * S::STAGES * 2 * S::TILE : 1];
    __shared__ uint32_t real[ATTEND_WARPS * S::STAGES];
    attend_enter();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    A at(cache, a, book, ring, scales, real);
    int64_t shared = 0, own = 0;
    for (int t0 = 0; t0 < a.n_tokens; t0 += ATTEND_THREADS) {
        const int t = t0 + (int)threadIdx.x;
        int64_t n = 0;
        bool nothing = false, without = false, sees = false;       // of this block's: no row; no pairs
        if (t < a.n_tokens) {
            const Seen r = seen_by(a, cache, t);
            const bool mine = t % gridDim.x == blockIdx.x;
            sees = r.end > 0;
            nothing = !sees && mine;
            book.seq[t] = r.s, book.end[t] = r.end;
            book.from[t] = GROUPED ? max(r.first, a.shared[t / a.group]) : r.first;
            if (!GROUPED) book.to[t] = r.end;
            const int32_t units = GROUPED || SHARED_WARPS == 0 ? at.own_units(t) : at.shared_units(t);
            if (units > 0)
                n = (int64_t)(GROUPED || SHARED_WARPS == 0 ? units + A::PAIR_COST : units + A::SHARED_PAIR_COST) *
                    (GROUPED || SHARED_WARPS == 0 ? cache.n_heads / a.together : cache.n_heads) * a.row_blocks;
            without = mine && units == 0;
        }
        uint32_t empty = __ballot_sync(0xFFFFFFFFu, without);
        const uint32_t seeing = __ballot_sync(0xFFFFFFFFu, sees);      // (a vote is no barrier: what others wrote is not read here)
        while (empty) {
            const int bit = __ffs(empty) - 1, i = t0 + warp * 32 + bit;
            empty &= empty - 1;
            for (int c = lane; c < cache.n_heads * a.row_blocks; c += 32)
                (SHARED_WARPS == 0 || GROUPED ? a.own_cuts : a.shared_cuts)[(int64_t)i * cache.n_heads * a.row_blocks + c] =
                    make_int2((seeing >> bit) & 1u ? 0 : -1, 0);
        }
        uint32_t which = __ballot_sync(0xFFFFFFFFu, nothing);
        while (which) {          // tokens without a row, by whole warps
            const int i = t0 + warp * 32 + __ffs(which) - 1;
            which &= which - 1;
            uint4 *row = reinterpret_cast<uint4 *>(a.out + i * a.out_stride);
            for (int c = lane; c < a.n_q_heads * cache.head_dim / 8; c += 32) row[c] = make_uint4(0, 0, 0, 0);
            if (a.lse)
                for (int c = lane; c < a.n_q_heads; c += 32) a.lse[(int64_t)i * a.n_q_heads + c] = NEG_INFINITY;
        }
        if (GROUPED || SHARED_WARPS == 0) {
            const int64_t before = sums_before(n, own, scan);
            if (t < a.n_tokens) book.upto[t] = before;
        } else {
            const int64_t before = sums_before(n, shared, scan);
            if (t < a.n_tokens) book.shared_upto[t] = before;
        }
    }
    if constexpr (GROUPED) {
        for (int g0 = 0; g0 < a.n_groups; g0 += ATTEND_THREADS) {
            const int g = g0 + (int)threadIdx.x;
            int64_t n = 0;
            if (g < a.n_groups) {
                book.to[g] = a.shared[g];
                const int32_t units = at.shared_units(g);
                if (units > 0) n = (int64_t)(units + A::SHARED_PAIR_COST) * a.shared_row_blocks * cache.n_heads;
                if (n == 0 && g % gridDim.x == blockIdx.x)
                    for (int c = 0; c < cache.n_heads * a.shared_row_blocks; ++c) a.shared_cuts[(int64_t)g * cache.n_heads * a.shared_row_blocks + c] = make_int2(0, 0);
            }
            const int64_t before = sums_before(n, shared, scan);
            if (g < a.n_groups) book.shared_upto[g] = before;
        }
    }
    // Blocks for the shared and for the tokens' own positions, by how many of them there are (in tiles of a head).
    int64_t blocks = GROUPED ? 0 : SHARED_WARPS > 0 ? (int64_t)gridDim.x : 0;
    if (GROUPED && shared > 0) {
        // (a shared unit takes 4/3 of the time that a warp's tiles of the same size take: 732 warps were done after 67 us, 452 after 53)
        const int64_t x = shared * ATTEND_WARPS * 4, y = own * a.together * 3;
        blocks = own == 0 ? (int64_t)gridDim.x : min(max(quotient((int64_t)gridDim.x * x, x + y), (int64_t)1), (int64_t)gridDim.x - 1);
    }
    at.shared_blocks = (int32_t)blocks;
    if (threadIdx.x == 0) {
        book.upto[a.n_tokens] = own, book.shared_upto[a.n_groups] = shared;
        book.shared.make(shared, at.shared_blocks);
    }
    if (threadIdx.x == 32) book.own.make(own, ((int32_t)gridDim.x - at.shared_blocks) * ATTEND_WARPS / a.together);
    __syncthreads();
    if constexpr (SHARED_WARPS > 0)
        if ((int)blockIdx.x < at.shared_blocks) {
            at.work_on_pairs();
            return;
        }
    if constexpr (GROUPED || SHARED_WARPS == 0) at.work_alone();
}

}  // namespace
