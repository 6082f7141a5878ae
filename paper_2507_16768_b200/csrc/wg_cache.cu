// What a paged cache holds (wg_rope_*, wg_kv_write, wg_kv_read of wg.h): a step's tokens rotated, quantised and put into
// their slots, and sequences read back.
#include <cmath>

#include "wg_cache.cuh"
#include "wg_host.h"

namespace {

constexpr int CACHE_THREADS = 256;
constexpr int READ_ROWS = 32;           // rows a block looks up together, at most

__device__ __forceinline__ void cache_enter() {
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    asm volatile("griddepcontrol.wait;" ::: "memory");
}

struct Frequencies {
    double f[WG_KV_MAX_HEAD_DIM / 2];
};

// Angles in fp64: at position 10^6 an fp32 angle is off by 0.03.  Made once for a model; one sincos an entry bounds it.
__global__ void __launch_bounds__(CACHE_THREADS)
rope_table_kernel(Frequencies freq, int32_t n_freq, int32_t n_pos, double magnitude, float *table) {
    cache_enter();
    const int64_t n = (int64_t)n_freq * n_pos;
    for (int64_t i = (int64_t)blockIdx.x * CACHE_THREADS + threadIdx.x; i < n; i += (int64_t)gridDim.x * CACHE_THREADS) {
        const int64_t p = i / n_freq;
        const int j = (int)(i - p * n_freq);
        double sine, cosine;
        sincos((double)p * freq.f[j], &sine, &cosine);
        float *row = table + p * 2 * n_freq;
        row[j] = (float)(cosine * magnitude);
        row[n_freq + j] = (float)(sine * magnitude);
    }
}

struct WriteArgs {
    const uint16_t *q, *k, *v;
    uint16_t *q_out;
    int64_t q_stride, k_stride, v_stride, q_out_stride;
    int32_t n_q_heads;
    const float *table;       // NULL: no rotation
    int32_t n_pos, rot, interleaved;
    const int64_t *slot;
    const int32_t *pos;
    int32_t *status;
    int32_t n_tokens;
    int32_t per, q_parts, k_parts;     // vectors of a lane group, and the groups of a token's queries and keys
    int32_t tokens;           // of a block
    Divisor lanes;            // of a vector, where they need not meet
};

// A lane has two chunks of eight dimensions of a vector, A and B, such that rotation stays within a lane: with pairs (i, i + rot / 2)
// they are rot / 2 apart, else neighbours.
struct Rotation {
    Two cosine[8], sine[8];   // of the words of A and B; sine with the sign that the partner enters with
    bool on;

    __device__ __forceinline__ void load(const WriteArgs &a, int32_t pos, int c) {
        on = c * 16 < a.rot;
        if (!on) return;
        const float *row = a.table + (int64_t)pos * a.rot + c * 8;
        float cs[8], sn[8];
#pragma unroll
        for (int i = 0; i < 8; i += 4) {
            const float4 x = *reinterpret_cast<const float4 *>(row + i), y = *reinterpret_cast<const float4 *>(row + a.rot / 2 + i);
            cs[i] = x.x, cs[i + 1] = x.y, cs[i + 2] = x.z, cs[i + 3] = x.w;
            sn[i] = y.x, sn[i + 1] = y.y, sn[i + 2] = y.z, sn[i + 3] = y.w;
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int u = 2 * (i & 3);
            cosine[i] = a.interleaved ? Two(cs[i], cs[i]) : Two(cs[u], cs[u + 1]);
            sine[i] = a.interleaved ? Two(-sn[i], sn[i]) : i < 4 ? Two(-sn[u], -sn[u + 1]) : Two(sn[u], sn[u + 1]);
        }
    }
    // (which of the products is rounded by itself is said in the header: results are the same whatever the layout)
    __device__ __forceinline__ void turn(Two (&y)[8], bool interleaved) const {
        Two partner[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float2 f = y[i].floats();
            partner[i] = interleaved ? Two(f.y, f.x) : y[i ^ 4];
        }
        if (on) {
#pragma unroll
            for (int i = 0; i < 8; ++i) y[i] = fused(y[i], cosine[i], partner[i] * sine[i]);
        }
    }
};

__device__ __forceinline__ uint32_t codes2(float2 f, E4m3) { return __nv_cvt_float2_to_fp8x2(f, __NV_SATFINITE, __NV_E4M3); }
__device__ __forceinline__ uint32_t codes2(float2 f, Int8) { return (uint32_t)(__float2int_rn(f.x) & 0xFF) | ((uint32_t)(__float2int_rn(f.y) & 0xFF) << 8); }

__device__ __forceinline__ float largest(float a, float b) {      // NaN if one of them is
    float y;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(y) : "f"(a), "f"(fabsf(b)));
    return y;
}

// The vector of a lane group, quantised: codes in the order of `y`, and its scale.
template <typename CODE, int LV>
__device__ __forceinline__ float quantise(const Two (&y)[8], uint32_t (&codes)[4], bool inside, uint32_t group) {
    float top = 0.0f;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const float2 f = y[i].floats();
        top = largest(largest(top, f.x), f.y);
    }
    if (!inside) top = 0.0f;
#pragma unroll
    for (int o = LV / 2; o > 0; o >>= 1) top = largest(top, __shfl_xor_sync(group, top, o));
    constexpr float LARGEST = std::is_same<CODE, E4m3>::value ? 448.0f : 127.0f;
    const bool finite = top < __uint_as_float(0x7F800000u), small = top < 0x1p-100f;
    const float mul = finite && !small ? __fdiv_rn(LARGEST, top) : 0.0f;
    const Two by(mul, mul);
#pragma unroll
    for (int i = 0; i < 4; ++i)
        codes[i] = finite ? codes2((y[2 * i] * by).floats(), CODE{}) | (codes2((y[2 * i + 1] * by).floats(), CODE{}) << 16) : 0u;
    return !finite ? __uint_as_float(0x7FC00000u) : small ? 1.0f : __fdiv_rn(top, LARGEST);
}

// A group of LV lanes (0: just as many as it takes, which do not meet) holds a vector, 16 elements a lane, and goes over some of a
// token's queries, keys or values with the token's angles in registers.  The groups of a warp have different tokens, all for the same.
//
// Memory, and instructions close behind.  12001 tokens with 32 + 16 heads of 128 into an 8-bit cache: 52 us, 5.1 TB/s, 0.77 of a copy's
// rate (into bf16: 50 us, 0.87); with a chunk a lane, partners by shuffle and single-number arithmetic 102 us.  Four vectors in
// flight: two 67 us; at most eight vectors a group: four 56, sixteen 52 (and 19 instead of 17 for 5000 tokens of 48 heads of 80).
// A step of four tokens: 2 us.
template <typename T, typename CODE, int LV>
__global__ void __launch_bounds__(CACHE_THREADS)
write_kernel(const __grid_constant__ CacheDev cache, const __grid_constant__ WriteArgs a) {
    cache_enter();
    constexpr int AHEAD = 4;             // vectors in flight
    constexpr bool NARROW = !std::is_same<CODE, T>::value;
    const int lane = threadIdx.x & 31, of = LV > 0 ? (int)threadIdx.x / (LV > 0 ? LV : 1) : (int)a.lanes.quotient(threadIdx.x);
    const int c = (int)threadIdx.x - of * (LV > 0 ? LV : (int)a.lanes.d);
    const uint32_t group = ((1u << LV) - 1u) << (lane & ~(LV - 1));
    const int64_t t = (int64_t)blockIdx.x * a.tokens + of;
    if (of >= a.tokens || t >= a.n_tokens) return;
    const int64_t slot = a.slot[t];
    const int32_t pos = a.table ? a.pos[t] : 0;
    const bool bad = slot < -1 || slot >= (int64_t)cache.n_blocks * cache.block.d || (slot >= 0 && a.table && (pos < 0 || pos >= a.n_pos));
    if (a.status && blockIdx.y == 0 && c == 0) a.status[t] = bad ? WG_ERR_ARG : WG_OK;
    if (bad || slot < 0) return;
    const int D = cache.head_dim;
    const bool inside = c * 16 < D;
    // what this group is for
    const int part = blockIdx.y;
    const bool queries = part < a.q_parts, values = part >= a.q_parts + a.k_parts;
    const int first = (part - (queries ? 0 : values ? a.q_parts + a.k_parts : a.q_parts)) * a.per;
    const int last = min(first + a.per, queries ? a.n_q_heads : cache.n_heads);
    const int half = a.interleaved ? 0 : a.rot / 16;
    const int at = (c < half ? c : 2 * c) * 8, far = (c < half ? half : 1) * 8;      // A (behind the pairs, 2 half + 2 (c - half)), and B from it
    const uint16_t *from = (queries ? a.q + t * a.q_stride : values ? a.v + t * a.v_stride : a.k + t * a.k_stride) + at;
    Rotation r;
    r.on = false;
    if (!values && a.table) r.load(a, pos, c);
    for (int h0 = first; h0 < last; h0 += AHEAD) {
        uint4 w[AHEAD][2];
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) {
            w[u][0] = w[u][1] = make_uint4(0, 0, 0, 0);
            if (h0 + u < last && inside) {
                const uint16_t *x = from + (h0 + u) * D;
                w[u][0] = __ldcs(reinterpret_cast<const uint4 *>(x)), w[u][1] = __ldcs(reinterpret_cast<const uint4 *>(x + far));
            }
        }
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) {
            const int h = h0 + u;
            if (h >= last) break;
            const uint32_t x[8] = {w[u][0].x, w[u][0].y, w[u][0].z, w[u][0].w, w[u][1].x, w[u][1].y, w[u][1].z, w[u][1].w};
            Two y[8];
            if (NARROW || !values) {
#pragma unroll
                for (int i = 0; i < 8; ++i) y[i] = Two(unpack(x[i], T{}));
                if (!values) r.turn(y, a.interleaved);
            }
            const int64_t row = slot * cache.n_heads + h;
            if constexpr (NARROW) {
                if (!queries) {
                    uint32_t codes[4];
                    const float scale = quantise<CODE, LV>(y, codes, inside, group);
                    if (c == 0) (values ? cache.v_scale : cache.k_scale)[row] = scale;
                    if (inside) {
                        char *to = (values ? cache.v : cache.k) + row * D + at;
                        *reinterpret_cast<uint2 *>(to) = make_uint2(codes[0], codes[1]);
                        *reinterpret_cast<uint2 *>(to + far) = make_uint2(codes[2], codes[3]);
                    }
                    continue;
                }
            }
            if (inside) {
                uint4 z[2] = {w[u][0], w[u][1]};
                if (!values) {
                    uint32_t p[8];
#pragma unroll
                    for (int i = 0; i < 8; ++i) p[i] = pack<T>(y[i].floats().x, y[i].floats().y);
                    z[0] = make_uint4(p[0], p[1], p[2], p[3]), z[1] = make_uint4(p[4], p[5], p[6], p[7]);
                }
                uint16_t *to = queries ? a.q_out + t * a.q_out_stride + h * D + at : reinterpret_cast<uint16_t *>(values ? cache.v : cache.k) + row * D + at;
                *reinterpret_cast<uint4 *>(to) = z[0];
                *reinterpret_cast<uint4 *>(to + far) = z[1];
            }
        }
    }
}

struct ReadArgs {
    const int32_t *table, *len, *cu;
    int64_t stride;
    int32_t max_blocks, n_seq, n_rows, rows_per_block;
    Divisor per_head;         // pieces of eight elements
    char *k_out, *v_out;
};

// Two codes of a word as fp32.
__device__ __forceinline__ Two codes_to_floats(uint32_t w, int pair, E4m3) {
    const uint32_t h = codes_to_half2(w, pair, E4m3{});
    return Two(unpack(h, __half{}));
}
__device__ __forceinline__ Two codes_to_floats(uint32_t w, int pair, Int8) {      // 0x4B000000 + u is 2^23 + u for a byte u = code + 128
    const uint32_t u = w ^ 0x80808080u;
    return Two(__uint_as_float(__byte_perm(u, 0x4B000000u, pair ? 0x7442 : 0x7440)), __uint_as_float(__byte_perm(u, 0x4B000000u, pair ? 0x7443 : 0x7441))) +
           Two(-8388736.0f, -8388736.0f);
}

template <typename CODE>
struct Eight {                       // eight elements as they are held
    using Word = uint2;
    static __device__ __forceinline__ void floats(uint2 w, float scale, float (&y)[8]) {
        const uint32_t x[2] = {w.x, w.y};
        const Two by(scale, scale);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float2 f = (codes_to_floats(x[i / 2], i & 1, CODE{}) * by).floats();
            y[2 * i] = f.x, y[2 * i + 1] = f.y;
        }
    }
};
template <typename T>
struct EightWide {
    using Word = uint4;
    static __device__ __forceinline__ void floats(uint4 w, float, float (&y)[8]) {
        const uint32_t x[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float2 f = unpack(x[i], T{});
            y[2 * i] = f.x, y[2 * i + 1] = f.y;
        }
    }
};
template <>
struct Eight<__nv_bfloat16> : EightWide<__nv_bfloat16> {};
template <>
struct Eight<__half> : EightWide<__half> {};

__device__ __forceinline__ void store8(char *to, const float (&y)[8], float) {
    reinterpret_cast<float4 *>(to)[0] = make_float4(y[0], y[1], y[2], y[3]);
    reinterpret_cast<float4 *>(to)[1] = make_float4(y[4], y[5], y[6], y[7]);
}
template <typename T>
__device__ __forceinline__ void store8(char *to, const float (&y)[8], T) {
    *reinterpret_cast<uint4 *>(to) = make_uint4(pack<T>(y[0], y[1]), pack<T>(y[2], y[3]), pack<T>(y[4], y[5]), pack<T>(y[6], y[7]));
}

// A block takes up to READ_ROWS rows of one plane: a lane per row finds its sequence and slot, then all warps copy.
// Memory: 40 ragged sequences up to 16384 positions, 8 heads of 128, int8 to bf16: 56 us, 5.8 TB/s, 0.89 of a copy's rate (with a
// division per piece and loads behind a branch 88 us).  700 positions: 2.9 us.
template <typename CODE, typename OUT>
__global__ void __launch_bounds__(CACHE_THREADS)
read_kernel(CacheDev cache, ReadArgs a) {
    cache_enter();
    using Word = typename Eight<CODE>::Word;
    constexpr bool NARROW = sizeof(Word) == 8;
    constexpr int AHEAD = 4;
    __shared__ int64_t slot_of[READ_ROWS];   // -1: zeros; -2: the row is none of a sequence's
    const bool values = blockIdx.y != 0;
    char *out = values ? a.v_out : a.k_out;
    if (!out) return;
    const int row0 = (int)((int64_t)blockIdx.x * a.rows_per_block), rows = min(a.rows_per_block, a.n_rows - row0);
    if ((int)threadIdx.x < rows) {
        const int row = row0 + (int)threadIdx.x;
        int lo = 0, hi = a.n_seq;            // the last s with cu[s] <= row
        while (hi - lo > 1) {
            const int mid = (lo + hi) >> 1;
            if (a.cu[mid] <= row) lo = mid; else hi = mid;
        }
        const int64_t p = (int64_t)row - a.cu[lo];
        int64_t slot = -2;
        if (p >= 0 && p < a.len[lo] && row < a.cu[lo + 1]) {
            const int64_t col = cache.block.quotient((uint32_t)p);
            const int32_t block = col < a.max_blocks ? a.table[lo * a.stride + col] : -1;
            slot = block < 0 || block >= cache.n_blocks ? -1 : (int64_t)block * cache.block.d + (p - col * cache.block.d);
        }
        slot_of[threadIdx.x] = slot;
    }
    __syncthreads();
    const char *plane = values ? cache.v : cache.k;
    const float *scales = values ? cache.v_scale : cache.k_scale;
    const int per_head = cache.head_dim / 8, per_row = cache.n_heads * per_head;
    // a thread goes from piece to piece, CACHE_THREADS apart, without dividing
    const int down = CACHE_THREADS / per_row, right = CACHE_THREADS - down * per_row;
    int row = (int)threadIdx.x / per_row, at = (int)threadIdx.x - row * per_row;
    char *to = out + ((int64_t)row0 * per_row + threadIdx.x) * (8 * (int64_t)sizeof(OUT));
    const auto take = [&](auto many) {
        constexpr int N = decltype(many)::value;
        Word w[N];
        float scale[N];
        int64_t slot[N];
#pragma unroll
        for (int u = 0; u < N; ++u) {
            slot[u] = slot_of[row];
            const int64_t from = max(slot[u], (int64_t)0);       // (something in any case: branches would keep the loads apart)
            w[u] = __ldcs(reinterpret_cast<const Word *>(plane + (from * per_row + at) * (int64_t)sizeof(Word)));
            scale[u] = 0.0f;
            if constexpr (NARROW) scale[u] = scales[from * cache.n_heads + a.per_head.quotient((uint32_t)at)];
            row += down, at += right;
            if (at >= per_row) at -= per_row, ++row;
        }
#pragma unroll
        for (int u = 0; u < N; ++u) {
            float y[8];
            Eight<CODE>::floats(w[u], scale[u], y);
#pragma unroll
            for (int i = 0; i < 8; ++i) y[i] = slot[u] < 0 ? 0.0f : y[i];
            if (slot[u] != -2) store8(to, y, OUT{});
            to += CACHE_THREADS * (8 * (int64_t)sizeof(OUT));
        }
    };
    while (row + (AHEAD - 1) * (down + (right != 0)) < rows) take(std::integral_constant<int, AHEAD>{});
    while (row < rows) take(std::integral_constant<int, 1>{});
}

template <typename T, typename CODE>
int32_t launch_write(const CacheDev &c, WriteArgs &a, cudaStream_t st) {
    const int heads = a.n_q_heads + 2 * c.n_heads;
    constexpr bool NARROW = !std::is_same<CODE, T>::value;
    const int lanes = !NARROW ? c.head_dim / 16 : c.head_dim <= 64 ? 4 : c.head_dim <= 128 ? 8 : 16;
    // as few vectors a group as the GPU has room for groups at once (768 threads an SM), and no more than 8: one for a step of few tokens
    const int64_t room = (int64_t)sm_count() * 768 / lanes;
    int64_t per = ((int64_t)a.n_tokens * heads + room - 1) / room;
    per = per < 1 ? 1 : per > 8 ? 8 : per;
    if ((heads + per - 1) / per + 3 > 65535) per = 8;
    a.per = (int)per;
    a.q_parts = (int)((a.n_q_heads + per - 1) / per), a.k_parts = (int)((c.n_heads + per - 1) / per);
    a.tokens = CACHE_THREADS / lanes, a.lanes = Divisor::of((uint32_t)lanes);
    const dim3 grid((unsigned)(((int64_t)a.n_tokens + a.tokens - 1) / a.tokens), (unsigned)(a.q_parts + 2 * a.k_parts));
    if constexpr (!NARROW) {
        WG_CUDA(launch_pdl(write_kernel<T, CODE, 0>, grid, dim3(CACHE_THREADS), st, c, a));
    } else {
        if (lanes == 4)
            WG_CUDA(launch_pdl(write_kernel<T, CODE, 4>, grid, dim3(CACHE_THREADS), st, c, a));
        else if (lanes == 8)
            WG_CUDA(launch_pdl(write_kernel<T, CODE, 8>, grid, dim3(CACHE_THREADS), st, c, a));
        else
            WG_CUDA(launch_pdl(write_kernel<T, CODE, 16>, grid, dim3(CACHE_THREADS), st, c, a));
    }
    WG_LAUNCHED();
    return WG_OK;
}

template <typename T>
int32_t launch_write_as(const CacheDev &c, int32_t storage, WriteArgs &a, cudaStream_t st) {
    if (storage == WG_KV_E4M3) return launch_write<T, E4m3>(c, a, st);
    if (storage == WG_KV_INT8) return launch_write<T, Int8>(c, a, st);
    return launch_write<T, T>(c, a, st);
}

template <typename CODE>
int32_t launch_read(const CacheDev &c, const ReadArgs &a, int32_t dtype, cudaStream_t st) {
    const dim3 grid((unsigned)(((int64_t)a.n_rows + a.rows_per_block - 1) / a.rows_per_block), 2);
    if (dtype == WG_DTYPE_BF16)
        WG_CUDA(launch_pdl(read_kernel<CODE, __nv_bfloat16>, grid, dim3(CACHE_THREADS), st, c, a));
    else if (dtype == WG_DTYPE_FP16)
        WG_CUDA(launch_pdl(read_kernel<CODE, __half>, grid, dim3(CACHE_THREADS), st, c, a));
    else
        WG_CUDA(launch_pdl(read_kernel<CODE, float>, grid, dim3(CACHE_THREADS), st, c, a));
    WG_LAUNCHED();
    return WG_OK;
}

}  // namespace

extern "C" {

int32_t wg_rope_frequencies(int32_t rot_dim, double base, double factor, double original, double low, double high, double *freq) {
    if (!freq || rot_dim < 2 || rot_dim % 2 || rot_dim > WG_KV_MAX_HEAD_DIM) return WG_ERR_ARG;
    if (!(base > 0.0) || !(factor > 0.0) || !std::isfinite(base) || !std::isfinite(factor)) return WG_ERR_ARG;
    if (!(original >= 0.0) || !std::isfinite(original)) return WG_ERR_ARG;
    if (original > 0.0 && (!(low >= 0.0) || !(high > low) || !std::isfinite(high))) return WG_ERR_ARG;
    for (int32_t i = 0; i < rot_dim / 2; ++i) {
        const double f = std::pow(base, -2.0 * i / rot_dim);
        double keep = 0.0;
        if (original > 0.0) {
            const double turns = original * f / 6.283185307179586476925;
            keep = (turns - low) / (high - low);
            keep = keep < 0.0 ? 0.0 : keep > 1.0 ? 1.0 : keep;
        }
        freq[i] = factor == 1.0 ? f : f * (keep + (1.0 - keep) / factor);
    }
    return WG_OK;
}

int32_t wg_rope_table(const double *freq, int32_t n_freq, int32_t n_pos, double magnitude, float *table, void *stream) {
    NvtxRange nvtx_range("wg_rope_table");
    if (!freq || !table || n_freq < 1 || n_freq > WG_KV_MAX_HEAD_DIM / 2 || n_pos < 1) return WG_ERR_ARG;
    Frequencies f{};
    for (int32_t i = 0; i < n_freq; ++i) f.f[i] = freq[i];
    const int64_t blocks = ((int64_t)n_freq * n_pos + CACHE_THREADS - 1) / CACHE_THREADS, most = (int64_t)sm_count() * 64;
    WG_CUDA(launch_pdl(rope_table_kernel, dim3((unsigned)(blocks < most ? blocks : most)), dim3(CACHE_THREADS),
                       static_cast<cudaStream_t>(stream), f, n_freq, n_pos, magnitude, table));
    WG_LAUNCHED();
    return WG_OK;
}

int32_t wg_kv_write(const wg_kv_cache *cache, const void *k, int64_t k_stride, const void *v, int64_t v_stride, const void *q,
                    int64_t q_stride, void *q_out, int64_t q_out_stride, int32_t n_q_heads, int32_t dtype, const wg_rope *rope,
                    const int64_t *slot, const int32_t *pos, int32_t n_tokens, int32_t *status, void *stream) {
    NvtxRange nvtx_range("wg_kv_write");
    if (!cache_ok(cache) || n_tokens < 0 || n_q_heads < 0 || n_q_heads > 65535) return WG_ERR_ARG;
    if (dtype != WG_DTYPE_BF16 && dtype != WG_DTYPE_FP16) return WG_ERR_ARG;
    if (cache->storage <= WG_KV_FP16 && (cache->storage == WG_KV_FP16) != (dtype == WG_DTYPE_FP16)) return WG_ERR_ARG;
    if (rope && (!rope->table || ((uintptr_t)rope->table & 15) || rope->n_pos < 1 || rope->rot_dim < 16 || rope->rot_dim % 16 ||
                 rope->rot_dim > cache->head_dim))
        return WG_ERR_ARG;
    if (n_tokens == 0) return WG_OK;                    // (arrays of nothing may have no address)
    if ((q != nullptr) != (q_out != nullptr) || (q != nullptr) != (n_q_heads > 0)) return WG_ERR_ARG;
    const int64_t width = (int64_t)cache->n_heads * cache->head_dim, q_width = (int64_t)n_q_heads * cache->head_dim;
    if (!rows_ok(k, k_stride, width) || !rows_ok(v, v_stride, width) || !slot || (rope && !pos)) return WG_ERR_ARG;
    if (q && (!rows_ok(q, q_stride, q_width) || !rows_ok(q_out, q_out_stride, q_width))) return WG_ERR_ARG;
    WriteArgs a{};
    a.q = static_cast<const uint16_t *>(q), a.k = static_cast<const uint16_t *>(k), a.v = static_cast<const uint16_t *>(v);
    a.q_out = static_cast<uint16_t *>(q_out);
    a.q_stride = q_stride, a.k_stride = k_stride, a.v_stride = v_stride, a.q_out_stride = q_out_stride;
    a.n_q_heads = n_q_heads;
    if (rope) a.table = rope->table, a.n_pos = rope->n_pos, a.rot = rope->rot_dim, a.interleaved = rope->interleaved != 0;
    a.slot = slot, a.pos = pos, a.status = status, a.n_tokens = n_tokens;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    return dtype == WG_DTYPE_BF16 ? launch_write_as<__nv_bfloat16>(cache_dev(cache), cache->storage, a, st)
                                  : launch_write_as<__half>(cache_dev(cache), cache->storage, a, st);
}

int32_t wg_kv_read(const wg_kv_cache *cache, const int32_t *table, int64_t table_stride, int32_t max_blocks, const int32_t *len,
                   int32_t n_seq, const int32_t *cu, void *k_out, void *v_out, int32_t dtype, int32_t n_rows, void *stream) {
    NvtxRange nvtx_range("wg_kv_read");
    if (!cache_ok(cache) || !table || max_blocks < 1 || table_stride < max_blocks || !len || !cu || n_seq < 1 || n_rows < 0)
        return WG_ERR_ARG;
    if (dtype != WG_DTYPE_BF16 && dtype != WG_DTYPE_FP16 && dtype != WG_DTYPE_FP32) return WG_ERR_ARG;
    if ((((uintptr_t)k_out | (uintptr_t)v_out) & 15) != 0) return WG_ERR_ARG;
    if (n_rows == 0 || (!k_out && !v_out)) return WG_OK;
    ReadArgs a{table, len, cu, table_stride, max_blocks, n_seq, n_rows, 0, Divisor::of((uint32_t)cache->head_dim / 8), static_cast<char *>(k_out),
               static_cast<char *>(v_out)};
    // rows of a block: enough blocks for the GPU, and then enough rows that their look-up is shared
    const int64_t spread = (int64_t)n_rows * 2 / (sm_count() * 8);
    a.rows_per_block = spread < 2 ? 2 : spread > READ_ROWS ? READ_ROWS : (int32_t)spread;
    const CacheDev c = cache_dev(cache);
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    switch (cache->storage) {
        case WG_KV_BF16: return launch_read<__nv_bfloat16>(c, a, dtype, st);
        case WG_KV_FP16: return launch_read<__half>(c, a, dtype, st);
        case WG_KV_E4M3: return launch_read<E4m3>(c, a, dtype, st);
        default: return launch_read<Int8>(c, a, dtype, st);
    }
}

}  // extern "C"
