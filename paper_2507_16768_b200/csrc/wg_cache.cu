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

// Angles in fp64: at position 10^6 an fp32 angle is off by 0.03.  Made once for a model.
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
    int32_t parts, per_part;  // a token's vectors are dealt out to `parts` lane groups
};

// Eight elements of a vector, rotated: those of chunk c, held by lane c of a group.
struct Rotation {
    float cosine[8], sine[8];   // (sine: with the sign that the element's partner enters with)
    int hc;                     // chunks of half the rotated part; 0: interleaved
    bool on;

    __device__ __forceinline__ void load(const WriteArgs &a, int32_t pos, int c) {
        on = a.table && c * 8 < a.rot;
        hc = a.interleaved ? 0 : a.rot / 16;
        if (!on) return;
        const float *row = a.table + (int64_t)pos * a.rot;
        if (hc == 0) {
            const float4 x = *reinterpret_cast<const float4 *>(row + c * 4), y = *reinterpret_cast<const float4 *>(row + a.rot / 2 + c * 4);
            const float cs[4] = {x.x, x.y, x.z, x.w}, sn[4] = {y.x, y.y, y.z, y.w};
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                cosine[i] = cs[i / 2];
                sine[i] = i & 1 ? sn[i / 2] : -sn[i / 2];
            }
        } else {
            const float *at = row + (c < hc ? c : c - hc) * 8;
#pragma unroll
            for (int i = 0; i < 8; i += 4) {
                const float4 x = *reinterpret_cast<const float4 *>(at + i), y = *reinterpret_cast<const float4 *>(at + a.rot / 2 + i);
                const float cs[4] = {x.x, x.y, x.z, x.w}, sn[4] = {y.x, y.y, y.z, y.w};
#pragma unroll
                for (int u = 0; u < 4; ++u) {
                    cosine[i + u] = cs[u];
                    sine[i + u] = c < hc ? -sn[u] : sn[u];
                }
            }
        }
    }

    // Every product is rounded by itself, as the header says: a fused multiply-add would round one of the two.
    template <typename T, int LG>
    __device__ __forceinline__ void turn(uint4 w, float (&y)[8], int c, uint32_t group) const {
        const uint32_t x[4] = {w.x, w.y, w.z, w.w};
        uint32_t other[4] = {x[0], x[1], x[2], x[3]};
        if (hc != 0) {
            const int from = c < hc ? c + hc : c < 2 * hc ? c - hc : c;
#pragma unroll
            for (int i = 0; i < 4; ++i) other[i] = __shfl_sync(group, x[i], from, LG);
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float2 own = unpack(x[i], T{}), partner = unpack(other[i], T{});
            if (!on) {
                y[2 * i] = own.x, y[2 * i + 1] = own.y;
                continue;
            }
            const float p0 = hc == 0 ? own.y : partner.x, p1 = hc == 0 ? own.x : partner.y;
            y[2 * i] = __fadd_rn(__fmul_rn(own.x, cosine[2 * i]), __fmul_rn(p0, sine[2 * i]));
            y[2 * i + 1] = __fadd_rn(__fmul_rn(own.y, cosine[2 * i + 1]), __fmul_rn(p1, sine[2 * i + 1]));
        }
    }
};

template <typename T>
__device__ __forceinline__ uint4 pack8(const float (&y)[8]) {
    return make_uint4(pack<T>(y[0], y[1]), pack<T>(y[2], y[3]), pack<T>(y[4], y[5]), pack<T>(y[6], y[7]));
}

__device__ __forceinline__ uint32_t codes4(float a, float b, float c, float d, E4m3) {
    const uint32_t lo = __nv_cvt_float2_to_fp8x2(make_float2(a, b), __NV_SATFINITE, __NV_E4M3);
    const uint32_t hi = __nv_cvt_float2_to_fp8x2(make_float2(c, d), __NV_SATFINITE, __NV_E4M3);
    return lo | (hi << 16);
}
__device__ __forceinline__ uint32_t codes4(float a, float b, float c, float d, Int8) {
    return (uint32_t)(__float2int_rn(a) & 0xFF) | ((uint32_t)(__float2int_rn(b) & 0xFF) << 8) |
           ((uint32_t)(__float2int_rn(c) & 0xFF) << 16) | ((uint32_t)__float2int_rn(d) << 24);
}

// The vector of a lane group, quantised into `codes` (row of head_dim bytes) and `scale`.
template <typename CODE, int LG>
__device__ __forceinline__ void quantise(const float (&y)[8], char *codes, float *scale, int c, bool inside, uint32_t group) {
    // as whole numbers magnitudes have the order of their values, with infinity and NaN above them
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) top = max(top, __float_as_uint(y[i]) & 0x7FFFFFFFu);
    if (!inside) top = 0;
#pragma unroll
    for (int o = LG / 2; o > 0; o >>= 1) top = max(top, __shfl_xor_sync(group, top, o));
    constexpr float LARGEST = sizeof(CODE) && std::is_same<CODE, E4m3>::value ? 448.0f : 127.0f;
    const float x = __uint_as_float(top);
    const bool finite = top < 0x7F800000u, small = x < 0x1p-100f;
    const float mul = finite && !small ? __fdiv_rn(LARGEST, x) : 0.0f;
    if (c == 0) *scale = !finite ? __uint_as_float(0x7FC00000u) : small ? 1.0f : __fdiv_rn(x, LARGEST);
    if (!inside) return;
    uint2 w = make_uint2(0, 0);
    if (finite)
        w = make_uint2(codes4(y[0] * mul, y[1] * mul, y[2] * mul, y[3] * mul, CODE{}),
                       codes4(y[4] * mul, y[5] * mul, y[6] * mul, y[7] * mul, CODE{}));
    *reinterpret_cast<uint2 *>(codes + c * 8) = w;
}

// A group of LG lanes holds a vector, eight elements a lane, and goes over its share of a token's vectors (queries, keys,
// values) with the token's angles in registers.
template <typename T, typename CODE, int LG>
__global__ void __launch_bounds__(CACHE_THREADS)
write_kernel(CacheDev cache, WriteArgs a) {
    cache_enter();
    constexpr int AHEAD = 4;             // vectors in flight
    constexpr bool NARROW = !std::is_same<CODE, T>::value;
    const int lane = threadIdx.x & 31, c = lane & (LG - 1);
    const uint32_t group = (LG == 32 ? 0xFFFFFFFFu : ((1u << LG) - 1u) << (lane & ~(LG - 1)));
    const int64_t id = ((int64_t)blockIdx.x * CACHE_THREADS + threadIdx.x) / LG;
    const int64_t t = id / a.parts;
    if (t >= a.n_tokens) return;
    const int part = (int)(id - t * a.parts);
    const int64_t slot = a.slot[t];
    const int32_t pos = a.table ? a.pos[t] : 0;
    const bool bad = slot < -1 || slot >= (int64_t)cache.n_blocks * cache.block.d || (slot >= 0 && a.table && (pos < 0 || pos >= a.n_pos));
    if (a.status && part == 0 && c == 0) a.status[t] = bad ? WG_ERR_ARG : WG_OK;
    if (bad || slot < 0) return;
    const bool inside = c * 8 < cache.head_dim;
    Rotation r;
    r.load(a, pos, c);
    const int n_heads = cache.n_heads, D = cache.head_dim, n = a.n_q_heads + 2 * n_heads;
    const int last = min(n, (part + 1) * a.per_part);
    for (int h0 = part * a.per_part; h0 < last; h0 += AHEAD) {
        uint4 w[AHEAD];
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) {
            const int h = h0 + u, hk = h - a.n_q_heads, hv = hk - n_heads;
            const uint16_t *from = hk < 0 ? a.q + t * a.q_stride + (int64_t)h * D : hv < 0 ? a.k + t * a.k_stride + (int64_t)hk * D
                                                                                          : a.v + t * a.v_stride + (int64_t)hv * D;
            w[u] = make_uint4(0, 0, 0, 0);
            if (h < last && inside) w[u] = *reinterpret_cast<const uint4 *>(from + c * 8);
        }
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) {
            const int h = h0 + u, hk = h - a.n_q_heads, hv = hk - n_heads;
            if (h >= last) break;
            float y[8];
            if (hv < 0) {
                r.turn<T, LG>(w[u], y, c, group);
            } else if constexpr (NARROW) {
                const uint32_t x[4] = {w[u].x, w[u].y, w[u].z, w[u].w};
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float2 f = unpack(x[i], T{});
                    y[2 * i] = f.x, y[2 * i + 1] = f.y;
                }
            }
            if (hk < 0) {
                if (inside) *reinterpret_cast<uint4 *>(a.q_out + t * a.q_out_stride + (int64_t)h * D + c * 8) = pack8<T>(y);
                continue;
            }
            const int64_t row = slot * n_heads + (hv < 0 ? hk : hv);
            char *plane = hv < 0 ? cache.k : cache.v;
            if constexpr (NARROW) {
                quantise<CODE, LG>(y, plane + row * D, (hv < 0 ? cache.k_scale : cache.v_scale) + row, c, inside, group);
            } else if (inside) {
                *reinterpret_cast<uint4 *>(plane + (row * D + c * 8) * 2) = hv < 0 ? pack8<T>(y) : w[u];
            }
        }
    }
}

struct ReadArgs {
    const int32_t *table, *len, *cu;
    int64_t stride;
    int32_t max_blocks, n_seq, n_rows, rows_per_block;
    char *k_out, *v_out;
};

template <typename CODE>
struct Eight {                       // eight elements as they are held
    using Word = uint2;
    static __device__ __forceinline__ void floats(uint2 w, float scale, float (&y)[8]) {
        const uint32_t x[2] = {w.x, w.y};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float2 f = unpack(codes_to_half2(x[i / 2], i & 1, CODE{}), __half{});
            y[2 * i] = f.x * scale, y[2 * i + 1] = f.y * scale;
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
    *reinterpret_cast<uint4 *>(to) = pack8<T>(y);
}

// A block takes up to READ_ROWS rows of one plane: a lane per row finds its sequence and slot, then all warps copy.
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
    const int per_head = cache.head_dim / 8, per_row = cache.n_heads * per_head, n = rows * per_row;
    for (int i0 = threadIdx.x; i0 < n; i0 += AHEAD * CACHE_THREADS) {
        Word w[AHEAD];
        float scale[AHEAD];
        int64_t slot[AHEAD];
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) {
            const int i = i0 + u * CACHE_THREADS, row = i / per_row, at = i - row * per_row;
            slot[u] = i < n ? slot_of[row] : -2;
            w[u] = Word{};
            scale[u] = 0.0f;
            if (slot[u] < 0) continue;
            w[u] = __ldcs(reinterpret_cast<const Word *>(plane + (slot[u] * per_row + at) * (int64_t)sizeof(Word)));
            if constexpr (NARROW) scale[u] = scales[slot[u] * cache.n_heads + at / per_head];
        }
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) {
            if (slot[u] == -2) continue;
            float y[8];
            Eight<CODE>::floats(w[u], scale[u], y);
            store8(out + ((int64_t)row0 * per_row + i0 + u * CACHE_THREADS) * (8 * (int64_t)sizeof(OUT)), y, OUT{});
        }
    }
}

template <typename T, typename CODE>
int32_t launch_write(const CacheDev &c, WriteArgs &a, cudaStream_t st) {
    const int heads = a.n_q_heads + 2 * c.n_heads;
    const int lanes = c.head_dim <= 64 ? 8 : c.head_dim <= 128 ? 16 : 32;
    // as few vectors a group as the GPU has room for groups at once, and no more than 16: one for a step of few tokens
    const int64_t room = (int64_t)sm_count() * 2048 / lanes;
    int64_t per = ((int64_t)a.n_tokens * heads + room - 1) / room;
    per = per < 1 ? 1 : per > 16 ? 16 : per;
    a.parts = (int)((heads + per - 1) / per);
    a.per_part = (heads + a.parts - 1) / a.parts;
    const int64_t blocks = ((int64_t)a.n_tokens * a.parts * lanes + CACHE_THREADS - 1) / CACHE_THREADS;
    if (blocks > 0x7FFFFFFF) return WG_ERR_ARG;
    const dim3 grid((unsigned)blocks);
    if (lanes == 8)
        WG_CUDA(launch_pdl(write_kernel<T, CODE, 8>, grid, dim3(CACHE_THREADS), st, c, a));
    else if (lanes == 16)
        WG_CUDA(launch_pdl(write_kernel<T, CODE, 16>, grid, dim3(CACHE_THREADS), st, c, a));
    else
        WG_CUDA(launch_pdl(write_kernel<T, CODE, 32>, grid, dim3(CACHE_THREADS), st, c, a));
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
    if ((q != nullptr) != (q_out != nullptr) || (q != nullptr) != (n_q_heads > 0) || (q && !rope)) return WG_ERR_ARG;
    if (rope && (!rope->table || ((uintptr_t)rope->table & 15) || rope->n_pos < 1 || rope->rot_dim < 16 || rope->rot_dim % 16 ||
                 rope->rot_dim > cache->head_dim))
        return WG_ERR_ARG;
    if (n_tokens == 0) return WG_OK;
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
    ReadArgs a{table, len, cu, table_stride, max_blocks, n_seq, n_rows, 0, static_cast<char *>(k_out), static_cast<char *>(v_out)};
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
