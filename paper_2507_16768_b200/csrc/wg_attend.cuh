// Attention of single tokens over a paged cache (wg_kv_attend of wg.h).
//
// The work is memory: every key and value is read once, by one warp, for the handful of rows (a head's queries) that
// need it.  A unit is UNIT_TOKENS positions of one (token, key head); all units of a call, in order of tokens and heads, are
// dealt out to the blocks in equal contiguous shares, whatever the lengths.  What a block holds of one (token, head)
// is a segment; a token whose units went to several blocks is joined by the block that arrives last, from
// partial results in scratch, always in the order of positions.
//
// Within a block a warp has rings of tiles of its own, filled with cp.async, 16 positions each, and the usual running
// maximum and sum: for x = scale q.k and the maximum m so far, p = 2^(x - m), l = sum of p, o = sum of p v, all
// multiplied by 2^(m_old - m) when m grows.  Rows are the M of mma.m16n8k16.  Both products read their second
// operand with plain 16-byte loads: the order of a dot product's terms is free, so a lane takes eight neighbouring
// dimensions of a key instead of the instruction's scattered pairs (and the queries are loaded the same way), and of the
// values it takes the same eight dimensions of four positions and pairs them with byte permutes, which makes
// the columns of the result neighbouring dimensions too.
//
// 8-bit caches.  Codes are exact in fp16.  Queries enter in fp16, divided by a power of two per row (a query of 2^-14 of the
// row's largest loses its last bits: 2^-25 of the largest).  A key's scale multiplies the score.  A value's scale s cannot
// simply multiply p, which then might fall below fp16's range while it matters: with x' = x + log2 s and the maximum m taken
// over x', p' = 2^(x' - m) is at most 1 and largest where the result comes from, and l is the sum of 2^(x - m).  Scales
// below 2^-100 count as that, which keeps l below 2^100 times the number of positions.
#pragma once

#include <type_traits>

#include "wg_cache.cuh"

constexpr int MAX_GROUPS = 1024;        // groups of tokens of one launch: their prefix sums are in shared memory

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
    int32_t row_blocks;           // of 16 rows each, of one token and key head
    int32_t q_bf16;
    float scale;                  // times log2(e)
    // scratch
    int32_t *shared;              // [n_groups] positions from 0 on that all of a group see in the same blocks
    int64_t *units;               // [n_groups]
    float *parts;                 // two per block: a segment that begins with the block's share, and one that does not
    float *shared_rows;           // [n_tokens][n_q_heads]: results of shared pairs that one block did by itself
    float *private_rows;          // ... and of the same tokens' private pairs
    int32_t *arrived;             // zero between calls
};

namespace {

constexpr int ATTEND_WARPS = 4, ATTEND_THREADS = 32 * ATTEND_WARPS;
constexpr int UNIT_TOKENS = 64;         // positions of a unit: a tile for each warp
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

__device__ __forceinline__ int32_t units_of(int32_t first, int32_t end) {
    return first < end ? (int32_t)(((uint32_t)(end - first) + UNIT_TOKENS - 1) / UNIT_TOKENS) : 0;
}

__device__ __forceinline__ void store_nothing(const AttendArgs &a, const CacheDev &cache, int t, int at, int threads) {
    uint4 *row = reinterpret_cast<uint4 *>(a.out + t * a.out_stride);
    for (int i = at; i < a.n_q_heads * cache.head_dim / 8; i += threads) row[i] = make_uint4(0, 0, 0, 0);
    if (a.lse)
        for (int i = at; i < a.n_q_heads; i += threads) a.lse[(int64_t)t * a.n_q_heads + i] = NEG_INFINITY;
}

// A block per group of tokens: how far their tables agree, and the units that makes.
__global__ void __launch_bounds__(ATTEND_THREADS)
attend_plan_kernel(CacheDev cache, AttendArgs a, int32_t shared_row_blocks) {
    attend_enter();
    __shared__ Seen seen[WG_BEAM_MAX_BEAMS];
    __shared__ int32_t differs;
    const int g = blockIdx.x, t0 = g * a.group;
    if (threadIdx.x == 0) differs = 0x7FFFFFFF;
    if ((int)threadIdx.x < a.group) seen[threadIdx.x] = seen_by(a, cache, t0 + (int)threadIdx.x);
    __syncthreads();
    int leader = -1, end = 0x7FFFFFFF;
    for (int m = a.group - 1; m >= 0; --m)
        if (seen[m].end > 0) leader = m, end = min(end, seen[m].end);
    for (int m = 0; m < a.group && t0 + m < a.n_tokens; ++m)
        if (seen[m].end == 0) store_nothing(a, cache, t0 + m, threadIdx.x, ATTEND_THREADS);
    if (leader < 0 || a.window > 0) end = 0;
    if (end > 0) {
        const int cols = (int)cache.block.quotient((uint32_t)(end - 1)) + 1;
        const int32_t *mine = a.table + seen[leader].s * a.stride;
        for (int c0 = 0; c0 < cols; c0 += 4 * ATTEND_THREADS) {
            int at = 0x7FFFFFFF;
#pragma unroll
            for (int u = 3; u >= 0; --u) {
                const int c = c0 + u * ATTEND_THREADS + (int)threadIdx.x;
                if (c >= cols) continue;
                const int32_t b = mine[c];
                bool same = true;
                for (int m = leader + 1; m < a.group; ++m)
                    if (seen[m].end > 0 && seen[m].s != seen[leader].s) same &= a.table[seen[m].s * a.stride + c] == b;
                if (!same) at = c;
            }
            if (at < 0x7FFFFFFF) atomicMin(&differs, at);
            if (__syncthreads_or(at < 0x7FFFFFFF)) break;
        }
        if (differs < 0x7FFFFFFF) end = (int)min((int64_t)end, (int64_t)differs * cache.block.d);
    }
    if (threadIdx.x < 32) {
        int64_t n = 0;
        if ((int)threadIdx.x < a.group && seen[threadIdx.x].end > 0) {
            const Seen r = seen[threadIdx.x];
            n = (int64_t)units_of(max(r.first, end), r.end) * a.row_blocks;
        }
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) n += __shfl_xor_sync(0xFFFFFFFFu, n, o);
        if (threadIdx.x == 0) {
            a.shared[g] = end;
            a.units[g] = (n + (int64_t)units_of(0, end) * shared_row_blocks) * cache.n_heads;
        }
    }
}

// ---- pieces of the inner loop --------------------------------------------------------------------------------

__device__ __forceinline__ uint32_t shared_address(const void *p) { return (uint32_t)__cvta_generic_to_shared(p); }
__device__ __forceinline__ void copy16(uint32_t to, const void *from, bool real) {   // zeros where it is not
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(to), "l"(from), "r"(real ? 16 : 0) : "memory");
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

// KV: what the cache holds; DP: the head size, rounded up (dimensions beyond it are zeros).
template <typename KV, int DP>
struct Shape {
    static constexpr bool NARROW = std::is_same<KV, E4m3>::value || std::is_same<KV, Int8>::value;
    using Mma = typename std::conditional<std::is_same<KV, __nv_bfloat16>::value, __nv_bfloat16, __half>::type;
    static constexpr int BYTES = NARROW ? 1 : 2;
    static constexpr int CHUNKS = DP * BYTES / 16;          // 16-byte pieces of a vector
    static constexpr int PLANE = 16 * DP * BYTES;           // a tile of keys, or of values
    static constexpr int STAGE = 2 * PLANE;
    static constexpr int STAGES = 24576 / STAGE > 8 ? 8 : 24576 / STAGE < 3 ? 3 : 24576 / STAGE;
    static constexpr int SMEM = ATTEND_WARPS * STAGES * STAGE;
    static constexpr int BLOCKS = SMEM > 110 * 1024 ? 1 : 2;        // on an SM
    static constexpr int STEPS = DP / 16;                   // of the first product
    static constexpr int HALVES = DP / 64;                  // of the second, 64 columns each
    static constexpr int PITCH = DP + 4;                    // of a row of partial results in shared memory, in floats
    static_assert(16 * PITCH * 4 + 128 <= STAGES * STAGE, "a warp's partial result takes the place of its ring");

    // Where piece c of vector r lies in a tile.  Eight lanes read 128 bytes at a time: four pieces of two neighbouring keys, one
    // or two of four values two rows apart; the pieces are swapped about so that those lie in different banks.
    static __device__ __forceinline__ int key_at(int r, int c) {
        const int g = r * CHUNKS + c;
        return CHUNKS >= 8 ? (g ^ ((r & 1) << 2)) * 16 : g * 16;
    }
    static __device__ __forceinline__ int value_at(int r, int c) { return ((r * CHUNKS + c) ^ (r & 6)) * 16; }
};

// One row block's running results in a warp: lane holds rows lane / 4 and lane / 4 + 8.
template <int HALVES>
struct Running {
    float m[2], l[2];
    float o[HALVES][8][4];        // [.][d][.]: dimensions 64 half + 16 (lane % 4) + d and + 8 + d, of both rows
    __device__ __forceinline__ void reset() {
        m[0] = m[1] = NEG_INFINITY;
        l[0] = l[1] = 0.0f;
#pragma unroll
        for (int h = 0; h < HALVES; ++h)
#pragma unroll
            for (int d = 0; d < 8; ++d)
#pragma unroll
                for (int i = 0; i < 4; ++i) o[h][d][i] = 0.0f;
    }
};

// Queries of a warp's 16 rows as the first operand.
template <typename KV, int DP>
struct Queries {
    using S = Shape<KV, DP>;
    uint32_t a[S::STEPS][4];
    float factor[2];              // of the rows' scores

    // row: NULL for none; `inside`: head_dim
    __device__ __forceinline__ void load(const uint16_t *row0, const uint16_t *row1, int head_dim, bool bf16, float scale, int j) {
        const uint16_t *row[2] = {row0, row1};
        factor[0] = factor[1] = scale;
        if constexpr (!S::NARROW) {
#pragma unroll
            for (int kk = 0; kk < S::STEPS / 2; ++kk)
#pragma unroll
                for (int u = 0; u < 2; ++u) {
                    const int d = (kk * 4 + j) * 8;
                    const uint4 x = row[u] && d < head_dim ? *reinterpret_cast<const uint4 *>(row[u] + d) : make_uint4(0, 0, 0, 0);
                    a[2 * kk][u] = x.x, a[2 * kk][2 + u] = x.y, a[2 * kk + 1][u] = x.z, a[2 * kk + 1][2 + u] = x.w;
                }
        } else {
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                uint32_t top = 0;
#pragma unroll
                for (int kk = 0; kk < S::STEPS / 4; ++kk)
#pragma unroll
                    for (int half = 0; half < 2; ++half) {
                        const int d = (kk * 4 + j) * 16 + half * 8;
                        const uint4 x = row[u] && d < head_dim ? *reinterpret_cast<const uint4 *>(row[u] + d) : make_uint4(0, 0, 0, 0);
                        const uint32_t w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            // word i belongs to step half * 2 + i / 2 of the four, registers u and 2 + u in turn
                            a[kk * 4 + half * 2 + i / 2][(i & 1) * 2 + u] = w[i];
                            const float2 f = bf16 ? unpack(w[i], __nv_bfloat16{}) : unpack(w[i], __half{});
                            top = max(top, max(__float_as_uint(f.x) & 0x7FFFFFFFu, __float_as_uint(f.y) & 0x7FFFFFFFu));
                        }
                    }
                top = max(top, __shfl_xor_sync(0xFFFFFFFFu, top, 1));
                top = max(top, __shfl_xor_sync(0xFFFFFFFFu, top, 2));
                const uint32_t e = min(max(top >> 23, 1u), 253u);
                const float down = __uint_as_float((254u - e) << 23);
                factor[u] = scale * __uint_as_float(e << 23);
#pragma unroll
                for (int st = 0; st < S::STEPS; ++st)
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        uint32_t &w = a[st][i * 2 + u];
                        const float2 f = bf16 ? unpack(w, __nv_bfloat16{}) : unpack(w, __half{});
                        w = pack<__half>(f.x * down, f.y * down);
                    }
            }
        }
    }
};

// 16 positions: keys at `keys`, values at `values` in shared memory; bit i of `real`: position i counts.  scales: 16 of
// keys, then 16 of values.
template <typename KV, int DP>
__device__ __forceinline__ void take_tile(Running<DP / 64> &run, const Queries<KV, DP> &q, uint32_t keys, uint32_t values,
                                          const float *scales, uint32_t real, int lane) {
    using S = Shape<KV, DP>;
    const int n = lane >> 2, j = lane & 3;
    float x[2][4] = {};
#pragma unroll
    for (int kk = 0; kk < S::CHUNKS / 4; ++kk)
#pragma unroll
        for (int nt = 0; nt < 2; ++nt) {
            const uint4 k = load16(keys + S::key_at(nt * 8 + n, kk * 4 + j));
            if constexpr (!S::NARROW) {
                multiply(x[nt], q.a[2 * kk], k.x, k.y, typename S::Mma{});
                multiply(x[nt], q.a[2 * kk + 1], k.z, k.w, typename S::Mma{});
            } else {
                const uint32_t w[4] = {k.x, k.y, k.z, k.w};
#pragma unroll
                for (int st = 0; st < 4; ++st)
                    multiply(x[nt], q.a[4 * kk + st], codes_to_half2(w[st], 0, KV{}), codes_to_half2(w[st], 1, KV{}), __half{});
            }
        }
    float up[2][2];                      // log2 of a value's scale
#pragma unroll
    for (int nt = 0; nt < 2; ++nt) {
        if constexpr (S::NARROW) {
            const float2 ks = *reinterpret_cast<const float2 *>(scales + nt * 8 + 2 * j);
            const float2 vs = *reinterpret_cast<const float2 *>(scales + 16 + nt * 8 + 2 * j);
            up[nt][0] = __log2f(vs.x < 0x1p-100f ? 0x1p-100f : vs.x);      // (a NaN stays one)
            up[nt][1] = __log2f(vs.y < 0x1p-100f ? 0x1p-100f : vs.y);
            x[nt][0] *= q.factor[0] * ks.x, x[nt][1] *= q.factor[0] * ks.y;
            x[nt][2] *= q.factor[1] * ks.x, x[nt][3] *= q.factor[1] * ks.y;
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) x[nt][i] *= q.factor[i >> 1];
            up[nt][0] = up[nt][1] = 0.0f;
        }
        if (real != 0xFFFFu) {
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (!((real >> (nt * 8 + 2 * j + (i & 1))) & 1u)) x[nt][i] = NEG_INFINITY;
        }
    }
    float base[2];
    bool grew = false;
    float shrink[2];
#pragma unroll
    for (int u = 0; u < 2; ++u) {
        float m = fmaxf(fmaxf(x[0][2 * u] + up[0][0], x[0][2 * u + 1] + up[0][1]), fmaxf(x[1][2 * u] + up[1][0], x[1][2 * u + 1] + up[1][1]));
        m = fmaxf(m, __shfl_xor_sync(0xFFFFFFFFu, m, 1));
        m = fmaxf(m, __shfl_xor_sync(0xFFFFFFFFu, m, 2));
        m = fmaxf(m, run.m[u]);
        base[u] = m == NEG_INFINITY ? 0.0f : m;
        shrink[u] = m > run.m[u] ? power2(run.m[u] - base[u]) : 1.0f;
        grew |= m > run.m[u];
        run.m[u] = m;
    }
    if (__any_sync(0xFFFFFFFFu, grew)) {
#pragma unroll
        for (int u = 0; u < 2; ++u) run.l[u] *= shrink[u];
#pragma unroll
        for (int h = 0; h < S::HALVES; ++h)
#pragma unroll
            for (int d = 0; d < 8; ++d)
#pragma unroll
                for (int i = 0; i < 4; ++i) run.o[h][d][i] *= shrink[i >> 1];
    }
    uint32_t p[4];
#pragma unroll
    for (int nt = 0; nt < 2; ++nt)
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            const float x0 = x[nt][2 * u] - base[u], x1 = x[nt][2 * u + 1] - base[u];
            float p0 = power2(x0), p1 = power2(x1);
            run.l[u] += p0 + p1;
            if constexpr (S::NARROW) p0 = power2(x0 + up[nt][0]), p1 = power2(x1 + up[nt][1]);
            p[nt * 2 + u] = pack<typename S::Mma>(p0, p1);
        }
#pragma unroll
    for (int h = 0; h < S::HALVES; ++h) {
        const int r[4] = {2 * j, 2 * j + 1, 2 * j + 8, 2 * j + 9};
        if constexpr (!S::NARROW) {
            uint4 v[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i] = load16(values + S::value_at(r[i], h * 8 + n));
            const uint32_t w[4][4] = {{v[0].x, v[0].y, v[0].z, v[0].w}, {v[1].x, v[1].y, v[1].z, v[1].w},
                                      {v[2].x, v[2].y, v[2].z, v[2].w}, {v[3].x, v[3].y, v[3].z, v[3].w}};
#pragma unroll
            for (int d = 0; d < 8; ++d) {
                const uint32_t sel = d & 1 ? 0x7632 : 0x5410;
                multiply(run.o[h][d], p, __byte_perm(w[0][d / 2], w[1][d / 2], sel), __byte_perm(w[2][d / 2], w[3][d / 2], sel),
                         typename S::Mma{});
            }
        } else {
            uint2 v[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i] = load8(values + S::value_at(r[i], h * 4 + n / 2) + (n & 1) * 8);
            const uint32_t w[4][2] = {{v[0].x, v[0].y}, {v[1].x, v[1].y}, {v[2].x, v[2].y}, {v[3].x, v[3].y}};
#pragma unroll
            for (int d = 0; d < 8; d += 2) {
                const uint32_t sel = d & 2 ? 0x7362 : 0x5140;
                const uint32_t b0 = __byte_perm(w[0][d / 4], w[1][d / 4], sel), b1 = __byte_perm(w[2][d / 4], w[3][d / 4], sel);
                multiply(run.o[h][d], p, codes_to_half2(b0, 0, KV{}), codes_to_half2(b1, 0, KV{}), __half{});
                multiply(run.o[h][d + 1], p, codes_to_half2(b0, 1, KV{}), codes_to_half2(b1, 1, KV{}), __half{});
            }
        }
    }
}

// ---- where things are ------------------------------------------------------------------------------------------

// Units of a call, dealt out: share w is [total * w / workers, total * (w + 1) / workers).
struct Deal {
    int64_t total;
    int32_t workers;
    __device__ __forceinline__ int64_t begin(int w) const { return total * w / workers; }
    __device__ __forceinline__ int owner(int64_t unit) const { return (int)(((unit + 1) * workers + total - 1) / total) - 1; }
    // the slot of scratch for worker w's segment of the units from `first` on
    __device__ __forceinline__ int64_t slot(int w, int64_t first) const { return 2 * (int64_t)w + (begin(w) >= first ? 0 : 1); }
};

// A run of units with the same rows and head.
struct Pair {
    int64_t first;            // unit
    int32_t units;
    int32_t token;            // of a private pair; the group's first of a shared one
    int32_t head, row_block;
    int32_t from, to, seq;    // positions, and a sequence whose table has them
    bool shared;
};

// The units of a group, in registers of a warp: lane m has member m's private pairs.
struct Group {
    Seen seen;
    int32_t units;            // per pair
    int64_t offset;           // of the member's first pair, from the group's first unit
    int32_t shared_to, shared_units;

    __device__ __forceinline__ void load(const AttendArgs &a, const CacheDev &cache, int g, int shared_row_blocks, int lane) {
        seen = Seen{0, 0, 0};
        if (lane < a.group) seen = seen_by(a, cache, g * a.group + lane);
        shared_to = a.shared[g];
        shared_units = units_of(0, shared_to);
        units = units_of(max(seen.first, shared_to), seen.end);
        const int64_t mine = (int64_t)units * a.row_blocks * cache.n_heads;
        int64_t upto = mine;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int64_t y = __shfl_up_sync(0xFFFFFFFFu, upto, o);
            if (lane >= o) upto += y;
        }
        offset = upto - mine + (int64_t)shared_units * shared_row_blocks * cache.n_heads;
    }
};

template <typename KV, int DP, int WMS, bool GROUPED>
struct Attend {
    using S = Shape<KV, DP>;
    static constexpr int ROWS = 16 * WMS;                       // of a shared pair
    static constexpr int PART_ROW = DP + 4;                     // floats of a row's partial result: o, m, l
    static constexpr int64_t PART = (int64_t)ROWS * PART_ROW;

    const CacheDev &cache;
    const AttendArgs &a;
    char *ring;
    float *scales;          // [warp][stage][32]
    uint32_t *real;         // [warp][stage]
    Deal deal;
    int32_t shared_row_blocks;

    // The token and query head of row i of a pair (token -1: none).
    __device__ __forceinline__ int row_of(const Pair &p, int i, int &head) const {
        if (!p.shared) {
            const int r = p.row_block * 16 + i;
            head = p.head * a.rows + r;
            return i < 16 && r < a.rows ? p.token : -1;
        }
        const int r = p.row_block * ROWS + i, m = r / a.rows;
        head = p.head * a.rows + (r - m * a.rows);
        return m < a.group && seen_by(a, cache, p.token + m).end > 0 ? p.token + m : -1;
    }

    // The warps that work on the same tiles: one, or all of the block.
    template <int WM>
    static __device__ __forceinline__ void stream_sync() {
        static_assert(WM == 1 || WM == ATTEND_WARPS, "");
        if constexpr (WM == 1)
            __syncwarp();
        else
            __syncthreads();
    }

    // Units [u0, u1) of a pair, written where they belong.  `whole`: they are all of the pair's.  `final`: and nothing
    // else belongs to its rows.
    template <int WM>
    __device__ __forceinline__ void segment(const Pair &pair, int64_t u0, int64_t u1, bool whole, bool final) {
        constexpr int STREAMS = ATTEND_WARPS / WM, STREAM_TOKENS = 16 * WM;
        const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, n = lane >> 2, j = lane & 3;
        const int stream = warp / WM, wm = warp % WM;
        const int from = pair.from + (int)(u0 - pair.first) * UNIT_TOKENS;
        const int to = (int)min((int64_t)pair.to, (int64_t)pair.from + (u1 - pair.first) * UNIT_TOKENS);
        const int tiles = (int)(((uint32_t)(to - from) + STREAM_TOKENS - 1) / STREAM_TOKENS);   // of all streams
        const int mine = tiles > stream ? (tiles - stream + STREAMS - 1) / STREAMS : 0;
        const int32_t *row = a.table + pair.seq * a.stride;
        const int es = S::BYTES, width = cache.head_dim * es;
        const int pieces = width / 16;
        char *const my_ring = ring + warp * S::STAGES * S::STAGE;                    // this warp's tiles
        char *const stream_ring = ring + stream * WM * S::STAGES * S::STAGE;

        const auto position = [&](int i) { return from + (i * STREAMS + stream) * STREAM_TOKENS + wm * 16 + (lane & 15); };
        const auto entry = [&](int i) {            // of the table; anything but a block where there is none
            const int p = position(i);
            return i < mine && p < to ? row[cache.block.quotient((uint32_t)p)] : -1;
        };
        const auto issue = [&](int i, int32_t block) {
            const int stage = i % S::STAGES;
            int64_t vec = -1;
            if ((uint32_t)block < (uint32_t)cache.n_blocks) {
                const uint32_t p = (uint32_t)position(i);
                vec = ((int64_t)block * cache.block.d + (p - cache.block.quotient(p) * cache.block.d)) * cache.n_heads + pair.head;
            }
            const uint32_t ok = __ballot_sync(0xFFFFFFFFu, vec >= 0) & 0xFFFFu;
            if (i < mine) {
                const uint32_t keys = shared_address(my_ring + stage * S::STAGE), values = keys + S::PLANE;
#pragma unroll
                for (int it = 0; it < S::CHUNKS / 2; ++it) {
                    const int r = (it * 32 + lane) / S::CHUNKS, c = lane % S::CHUNKS;
                    const int64_t v = __shfl_sync(0xFFFFFFFFu, vec, r);
                    const bool is = v >= 0 && c < pieces;
                    const int64_t off = is ? v * width + c * 16 : 0;
                    copy16(keys + S::key_at(r, c), cache.k + off, is);
                    copy16(values + S::value_at(r, c), cache.v + off, is);
                }
                if constexpr (S::NARROW)
                    copy4(shared_address(scales + (warp * S::STAGES + stage) * 32 + lane),
                          (lane < 16 ? cache.k_scale : cache.v_scale) + (vec < 0 ? 0 : vec), vec >= 0);
                if (lane == 0) real[warp * S::STAGES + stage] = ok;
            }
            asm volatile("cp.async.commit_group;" ::: "memory");
        };
        int32_t first_blocks[S::STAGES - 1];
#pragma unroll
        for (int i = 0; i < S::STAGES - 1; ++i) first_blocks[i] = entry(i);
        int32_t next = entry(S::STAGES - 1);
        Queries<KV, DP> q;
        {
            const uint16_t *rows[2];
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                int head;
                const int t = row_of(pair, wm * 16 + n + 8 * u, head);
                rows[u] = t < 0 ? nullptr : a.q + t * a.q_stride + (int64_t)head * cache.head_dim;
            }
#pragma unroll
            for (int i = 0; i < S::STAGES - 1; ++i) issue(i, first_blocks[i]);
            q.load(rows[0], rows[1], cache.head_dim, a.q_bf16, a.scale, j);
        }
        Running<S::HALVES> run;
        run.reset();
#pragma unroll 1
        for (int i = 0; i < mine; ++i) {
            asm volatile("cp.async.wait_group %0;" ::"n"(S::STAGES - 2) : "memory");
            stream_sync<WM>();
            // (the tile that was used last is free: all warps of the stream are past it)
            issue(i + S::STAGES - 1, next);
            next = entry(i + S::STAGES);
            const int stage = i % S::STAGES;
#pragma unroll 1
            for (int w = 0; w < WM; ++w) {
                const int of = stream * WM + w;
                const uint32_t ok = real[of * S::STAGES + stage];
                const uint32_t keys = shared_address(stream_ring + (w * S::STAGES + stage) * S::STAGE);
                if (ok)
                    take_tile<KV, DP>(run, q, keys, keys + S::PLANE, scales + (of * S::STAGES + stage) * 32, ok, lane);
            }
        }
        asm volatile("cp.async.wait_group 0;" ::: "memory");
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            run.l[u] += __shfl_xor_sync(0xFFFFFFFFu, run.l[u], 1);
            run.l[u] += __shfl_xor_sync(0xFFFFFFFFu, run.l[u], 2);
        }
        stream_sync<WM>();
        // every warp's results into its ring
        float *const part = reinterpret_cast<float *>(my_ring);
        float2 *const stats = reinterpret_cast<float2 *>(part + 16 * S::PITCH);
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            const int r = n + 8 * u;
            if (j == 0) stats[r] = make_float2(run.m[u], run.l[u]);
#pragma unroll
            for (int h = 0; h < S::HALVES; ++h)
#pragma unroll
                for (int half = 0; half < 2; ++half)
#pragma unroll
                    for (int d = 0; d < 8; d += 4)
                        *reinterpret_cast<float4 *>(part + r * S::PITCH + h * 64 + j * 16 + half * 8 + d) =
                            make_float4(run.o[h][d][2 * u + half], run.o[h][d + 1][2 * u + half], run.o[h][d + 2][2 * u + half],
                                        run.o[h][d + 3][2 * u + half]);
        }
        __syncthreads();
        // joined over the streams: a thread takes eight dimensions of a row
        const int n_rows = pair.shared ? STREAM_TOKENS : min(16, a.rows - pair.row_block * 16);
        float *const to_part = a.parts + deal.slot(blockIdx.x, pair.first) * PART;
        for (int i = threadIdx.x; i < n_rows * (DP / 8); i += ATTEND_THREADS) {
            const int r = i / (DP / 8), d = (i % (DP / 8)) * 8;
            const char *base = ring + (r / 16) * S::STAGES * S::STAGE;
            float m = NEG_INFINITY, l = 0.0f, y[8] = {};
            float2 st[STREAMS];
#pragma unroll
            for (int s = 0; s < STREAMS; ++s) {
                const float *of = reinterpret_cast<const float *>(base + s * WM * S::STAGES * S::STAGE);
                st[s] = reinterpret_cast<const float2 *>(of + 16 * S::PITCH)[r & 15];
                m = fmaxf(m, st[s].x);
            }
#pragma unroll
            for (int s = 0; s < STREAMS; ++s) {
                const float *of = reinterpret_cast<const float *>(base + s * WM * S::STAGES * S::STAGE) + (r & 15) * S::PITCH + d;
                const float w = st[s].x == NEG_INFINITY ? (st[s].y == 0.0f ? 0.0f : 1.0f) : power2(st[s].x - m);   // (a sum without maximum: NaN)
                l += st[s].y * w;
#pragma unroll
                for (int e = 0; e < 8; ++e) y[e] += of[e] * w;
            }
            int head, t = 0;
            if (whole) {
                t = row_of(pair, r, head);
                if (t < 0) continue;
            }
            if (final) {
                if (d < cache.head_dim) store_row<8>(t, head, d, m, l, y);
                continue;
            }
            float *to_row = whole ? (pair.shared ? a.shared_rows : a.private_rows) + ((int64_t)t * a.n_q_heads + head) * PART_ROW
                                  : to_part + r * PART_ROW;
            *reinterpret_cast<float4 *>(to_row + d) = make_float4(y[0], y[1], y[2], y[3]);
            *reinterpret_cast<float4 *>(to_row + d + 4) = make_float4(y[4], y[5], y[6], y[7]);
            if (d == 0) *reinterpret_cast<float2 *>(to_row + DP) = make_float2(m, l);
        }
    }

    template <int N>
    __device__ __forceinline__ void store_row(int t, int head, int d, float m, float l, const float (&y)[N]) {
        const float by = l == 0.0f ? 0.0f : 1.0f / l;
        uint32_t w[N / 2];
#pragma unroll
        for (int e = 0; e < N; e += 2) {
            const float y0 = l == 0.0f ? 0.0f : y[e] * by, y1 = l == 0.0f ? 0.0f : y[e + 1] * by;
            w[e / 2] = a.q_bf16 ? pack<__nv_bfloat16>(y0, y1) : pack<__half>(y0, y1);
        }
        uint16_t *to = a.out + t * a.out_stride + (int64_t)head * cache.head_dim + d;
        if constexpr (N == 8)
            *reinterpret_cast<uint4 *>(to) = make_uint4(w[0], w[1], w[2], w[3]);
        else if constexpr (N == 4)
            *reinterpret_cast<uint2 *>(to) = make_uint2(w[0], w[1]);
        else
            *reinterpret_cast<uint32_t *>(to) = w[0];
        if (a.lse && d == 0)
            a.lse[(int64_t)t * a.n_q_heads + head] = l == 0.0f ? NEG_INFINITY : (m + log2f(l)) * 0.693147180559945f;
    }

    // The partial results of a row that belong to one pair: those of `n` workers from w on, or of the only one.
    struct Pieces {
        int32_t n, w;
        int64_t first;        // the pair's
        const float *only;
    };

    __device__ __forceinline__ Pieces pieces_of(int64_t first, int32_t units, const float *only) const {
        if (units == 0) return {0, 0, 0, nullptr};
        const int w = deal.owner(first);
        return {deal.owner(first + units - 1) - w + 1, w, first, only};
    }
    __device__ __forceinline__ const float *piece(const Pieces &p, int i, int row) const {
        return p.n == 1 ? p.only : a.parts + deal.slot(p.w + i, p.first) * PART + row * PART_ROW;
    }

    // A row's partial results joined by a warp, x's (row rx of their slots) before z's.
    __device__ __forceinline__ void join_row(int t, int head, const Pieces &x, int rx, const Pieces &z, int rz, int lane) {
        constexpr int PER = DP / 32;
        const auto part = [&](int i) { return i < x.n ? piece(x, i, rx) : piece(z, i - x.n, rz); };
        const int n = x.n + z.n;
        float m = NEG_INFINITY, l = 0.0f, y[PER] = {};
        for (int i0 = 0; i0 < n; i0 += 32) {
            const int i = i0 + lane;
            float mi = NEG_INFINITY, li = 0.0f;
            if (i < n) {
                const float2 st = __ldcg(reinterpret_cast<const float2 *>(part(i) + DP));
                mi = st.x, li = st.y;
            }
            float top = mi;
#pragma unroll
            for (int o = 16; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, o));
            top = fmaxf(top, m);
            const float w = mi == NEG_INFINITY ? (li == 0.0f ? 0.0f : 1.0f) : power2(mi - top);   // (a sum without maximum: NaN)
            const float old = m == NEG_INFINITY ? (l == 0.0f ? 0.0f : 1.0f) : power2(m - top);
            float sum = li * w;
#pragma unroll
            for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xFFFFFFFFu, sum, o);
            l = l * old + sum;
            m = top;
#pragma unroll
            for (int e = 0; e < PER; ++e) y[e] *= old;
            const int here = min(32, n - i0);
#pragma unroll 4
            for (int k = 0; k < here; ++k) {
                const float by = __shfl_sync(0xFFFFFFFFu, w, k);
                const float *p = part(i0 + k) + lane * PER;
#pragma unroll
                for (int e = 0; e < PER; e += 2) {
                    const float2 f = __ldcg(reinterpret_cast<const float2 *>(p + e));
                    y[e] += f.x * by, y[e + 1] += f.y * by;
                }
            }
        }
        if (lane * PER < cache.head_dim) store_row<PER>(t, head, lane * PER, m, l, y);
    }

    // This block's part of a pair, or of all pairs of a group and head, is written.  Whoever is the last to say so of
    // `expected` joins them.
    __device__ __forceinline__ bool arrive(int64_t counter, int expected, int *flag) {
        __threadfence();
        __syncthreads();
        if (threadIdx.x == 0) {
            const int before = atomicAdd(a.arrived + counter, 1);
            const bool last = before == expected - 1;
            if (last) a.arrived[counter] = 0;
            *flag = last;
        }
        __syncthreads();
        const bool last = *flag != 0;
        if (last) __threadfence();
        return last;
    }
};

// Registers: 64 (o) + 32 (queries) + loads at 128 dimensions; two blocks of four warps on an SM.
template <typename KV, int DP, int WMS, bool GROUPED>
__global__ void __launch_bounds__(ATTEND_THREADS, Shape<KV, DP>::BLOCKS)
attend_kernel(const __grid_constant__ CacheDev cache, const __grid_constant__ AttendArgs a) {
    using S = Shape<KV, DP>;
    extern __shared__ __align__(128) char ring[];
    __shared__ int64_t upto[MAX_GROUPS + 1];      // units before a group
    __shared__ int64_t scan[ATTEND_WARPS];
    __shared__ float scales[S::NARROW ? ATTEND_WARPS * S::STAGES * 32 : 1];
    __shared__ uint32_t real[ATTEND_WARPS * S::STAGES];
    __shared__ int flag;
    attend_enter();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    int64_t total = 0;
    for (int g0 = 0; g0 < a.n_groups; g0 += ATTEND_THREADS) {
        const int g = g0 + (int)threadIdx.x;
        int64_t n = 0;
        if constexpr (GROUPED) {
            if (g < a.n_groups) n = a.units[g];
        } else {
            bool nothing = false;
            if (g < a.n_groups) {
                const Seen r = seen_by(a, cache, g);
                n = (int64_t)units_of(r.first, r.end) * a.row_blocks * cache.n_heads;
                nothing = r.end == 0 && g % gridDim.x == blockIdx.x;
            }
            uint32_t which = __ballot_sync(0xFFFFFFFFu, nothing);
            while (which) {
                const int i = __ffs(which) - 1;
                which &= which - 1;
                store_nothing(a, cache, g0 + warp * 32 + i, lane, 32);
            }
        }
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
        if (g < a.n_groups) upto[g] = before + x - n;
        __syncthreads();
    }
    if (threadIdx.x == 0) upto[a.n_groups] = total;
    __syncthreads();
    if (total == 0) return;
    const int32_t workers = (int32_t)min((int64_t)gridDim.x, total);
    if ((int)blockIdx.x >= workers) return;
    const int32_t shared_row_blocks = GROUPED ? (a.group * a.rows + 16 * WMS - 1) / (16 * WMS) : 0;
    Attend<KV, DP, WMS, GROUPED> at{cache, a, ring, scales, real, Deal{total, workers}, shared_row_blocks};
    int64_t u = at.deal.begin(blockIdx.x);
    const int64_t end = at.deal.begin(blockIdx.x + 1);
    int g = 0;
    {
        int lo = 0, hi = a.n_groups;              // the last g with upto[g] <= u
        while (hi - lo > 1) {
            const int mid = (lo + hi) >> 1;
            if (upto[mid] <= u) lo = mid; else hi = mid;
        }
        g = lo;
    }
#pragma unroll 1
    while (u < end) {
        while (upto[g + 1] <= u) ++g;
        const int64_t o = u - upto[g];
        Pair p{};
        Group group;
        if constexpr (GROUPED) {
            group.load(a, cache, g, shared_row_blocks, lane);
            const int64_t n_shared = (int64_t)group.shared_units * shared_row_blocks * cache.n_heads;
            if (o < n_shared) {
                const int i = (int)(o / group.shared_units);
                const uint32_t live = __ballot_sync(0xFFFFFFFFu, group.seen.end > 0);
                p.shared = true;
                p.first = upto[g] + (int64_t)i * group.shared_units;
                p.units = group.shared_units;
                p.token = g * a.group;
                p.head = i / shared_row_blocks, p.row_block = i % shared_row_blocks;
                p.from = 0, p.to = group.shared_to;
                p.seq = __shfl_sync(0xFFFFFFFFu, group.seen.s, __ffs(live) - 1);
            } else {
                const int64_t size = (int64_t)group.units * a.row_blocks * cache.n_heads;
                const int m = __ffs(__ballot_sync(0xFFFFFFFFu, o >= group.offset && o < group.offset + size)) - 1;
                const int32_t units = __shfl_sync(0xFFFFFFFFu, group.units, m);
                const int64_t off = __shfl_sync(0xFFFFFFFFu, group.offset, m);
                const int i = (int)((o - off) / units);
                p.first = upto[g] + off + (int64_t)i * units;
                p.units = units;
                p.token = g * a.group + m;
                p.head = i / a.row_blocks, p.row_block = i % a.row_blocks;
                p.from = max(__shfl_sync(0xFFFFFFFFu, group.seen.first, m), group.shared_to);
                p.to = __shfl_sync(0xFFFFFFFFu, group.seen.end, m);
                p.seq = __shfl_sync(0xFFFFFFFFu, group.seen.s, m);
            }
        } else {
            const Seen r = seen_by(a, cache, g);
            p.units = units_of(r.first, r.end);
            const int i = (int)(o / p.units);
            p.first = upto[g] + (int64_t)i * p.units;
            p.token = g;
            p.head = i / a.row_blocks, p.row_block = i % a.row_blocks;
            p.from = r.first, p.to = r.end, p.seq = r.s;
        }
        const int64_t stop = min(end, p.first + p.units);
        bool with_shared = false;
        if constexpr (GROUPED) with_shared = group.shared_to > 0;     // (then all of the group's pairs of a head are joined)
        const bool whole = u == p.first && stop == p.first + p.units, final = whole && !with_shared;
        if (GROUPED && p.shared)
            at.template segment<WMS>(p, u, stop, whole, final);
        else
            at.template segment<1>(p, u, stop, whole, final);
        if (!final && !with_shared) {
            const auto all = at.pieces_of(p.first, p.units, nullptr);
            if (at.arrive(((int64_t)p.token * cache.n_heads + p.head) * a.row_blocks + p.row_block, all.n, &flag)) {
                const int rows = min(16, a.rows - p.row_block * 16);
                for (int r = warp; r < rows; r += ATTEND_WARPS)
                    at.join_row(p.token, p.head * a.rows + p.row_block * 16 + r, all, r, {0, 0, 0, nullptr}, 0, lane);
            }
        }
        if constexpr (GROUPED) {
            if (with_shared) {
                const int64_t shared_first = upto[g] + (int64_t)p.head * shared_row_blocks * group.shared_units;
                const int64_t own_first = upto[g] + group.offset + (int64_t)p.head * a.row_blocks * group.units;   // (of the lane's member)
                int expected = 0, own = 0;
                for (int b = 0; b < shared_row_blocks; ++b)
                    expected += at.pieces_of(shared_first + (int64_t)b * group.shared_units, group.shared_units, nullptr).n;
                for (int b = 0; b < a.row_blocks; ++b) own += at.pieces_of(own_first + (int64_t)b * group.units, group.units, nullptr).n;
#pragma unroll
                for (int d = 16; d > 0; d >>= 1) own += __shfl_xor_sync(0xFFFFFFFFu, own, d);
                if (at.arrive(((int64_t)g * a.group * cache.n_heads + p.head) * a.row_blocks, expected + own, &flag)) {
                    for (int r = warp; r < a.group * a.rows; r += ATTEND_WARPS) {
                        const int m = r / a.rows, of = r - m * a.rows, t = g * a.group + m, head = p.head * a.rows + of;
                        const int64_t first = __shfl_sync(0xFFFFFFFFu, own_first, m);
                        const int32_t units = __shfl_sync(0xFFFFFFFFu, group.units, m);
                        if (__shfl_sync(0xFFFFFFFFu, group.seen.end, m) == 0) continue;
                        const int64_t row = ((int64_t)t * a.n_q_heads + head) * at.PART_ROW;
                        const int rb = r / at.ROWS;
                        at.join_row(t, head, at.pieces_of(shared_first + (int64_t)rb * group.shared_units, group.shared_units, a.shared_rows + row),
                                    r - rb * at.ROWS, at.pieces_of(first + (int64_t)(of / 16) * units, units, a.private_rows + row), of % 16, lane);
                    }
                }
            }
        }
        u = stop;
        __syncthreads();      // the rings are free again
    }
}

}  // namespace
