// What the kernels on a cache's contents share: element types, 8-bit codes, the cache as a kernel sees it.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_fp8.h>
#include <cuda_runtime.h>
#include <cstdint>

#include "wg.h"
#include "wg_divide.cuh"

struct CacheDev {
    char *k, *v;
    float *k_scale, *v_scale;
    int32_t n_blocks, n_heads, head_dim;
    Divisor block;        // tokens of a block
};

// A cache whose sizes and pointers the kernels can work with.
inline bool cache_ok(const wg_kv_cache *c) {
    if (!c || !c->k || !c->v || c->storage < WG_KV_BF16 || c->storage > WG_KV_INT8) return false;
    const bool narrow = c->storage >= WG_KV_E4M3;
    if (narrow != (c->k_scale != nullptr) || narrow != (c->v_scale != nullptr)) return false;
    if (c->n_blocks < 1 || c->n_blocks > (1 << 30) || c->block_size < 1 || c->block_size > (1 << 30)) return false;
    if ((int64_t)c->n_blocks * c->block_size >= (1ll << 32)) return false;      // (slots are counted in 32 bits)
    if (c->n_heads < 1 || c->n_heads > 1024 || c->head_dim < 16 || c->head_dim > WG_KV_MAX_HEAD_DIM || c->head_dim % 16) return false;
    return (((uintptr_t)c->k | (uintptr_t)c->v) & 15) == 0 && (((uintptr_t)c->k_scale | (uintptr_t)c->v_scale) & 3) == 0;
}

inline CacheDev cache_dev(const wg_kv_cache *c) {
    return {static_cast<char *>(c->k), static_cast<char *>(c->v), c->k_scale, c->v_scale, c->n_blocks, c->n_heads, c->head_dim,
            Divisor::of((uint32_t)c->block_size)};
}

// Rows of 16-bit elements that are read and written 16 bytes at a time.
inline bool rows_ok(const void *p, int64_t stride, int64_t width) {
    return p && ((uintptr_t)p & 15) == 0 && stride >= width && stride % 8 == 0;
}

__device__ __forceinline__ float2 unpack(uint32_t w, __nv_bfloat16) {
    return {__uint_as_float(w << 16), __uint_as_float(w & 0xFFFF0000u)};
}
__device__ __forceinline__ float2 unpack(uint32_t w, __half) { return __half22float2(*reinterpret_cast<__half2 *>(&w)); }

template <typename T>
__device__ __forceinline__ uint32_t pack(float a, float b);
template <>
__device__ __forceinline__ uint32_t pack<__nv_bfloat16>(float a, float b) {
    const __nv_bfloat162 x = __floats2bfloat162_rn(a, b);
    return *reinterpret_cast<const uint32_t *>(&x);
}
template <>
__device__ __forceinline__ uint32_t pack<__half>(float a, float b) {
    const __half2 x = __floats2half2_rn(a, b);
    return *reinterpret_cast<const uint32_t *>(&x);
}

// Two fp32 numbers that one instruction works on, each rounded by itself.
struct Two {
    uint64_t x;
    Two() = default;
    __device__ __forceinline__ Two(float a, float b) { asm("mov.b64 %0, {%1, %2};" : "=l"(x) : "f"(a), "f"(b)); }
    __device__ __forceinline__ Two(float2 f) : Two(f.x, f.y) {}
    __device__ __forceinline__ float2 floats() const {
        float2 f;
        asm("mov.b64 {%0, %1}, %2;" : "=f"(f.x), "=f"(f.y) : "l"(x));
        return f;
    }
};
__device__ __forceinline__ Two operator*(Two a, Two b) {
    Two y;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(y.x) : "l"(a.x), "l"(b.x));
    return y;
}
__device__ __forceinline__ Two operator+(Two a, Two b) {
    Two y;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(y.x) : "l"(a.x), "l"(b.x));
    return y;
}
__device__ __forceinline__ Two fused(Two a, Two b, Two c) {      // a b + c, rounded once
    Two y;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(y.x) : "l"(a.x), "l"(b.x), "l"(c.x));
    return y;
}

struct E4m3 {};
struct Int8 {};

// Two neighbouring codes of a word as a pair of fp16 (exact for both types).  `pair`: 0 or 1.
__device__ __forceinline__ uint32_t codes_to_half2(uint32_t w, int pair, E4m3) {
    uint32_t y;
    if (pair)
        asm("{ .reg .b16 lo, hi; mov.b32 {lo, hi}, %1; cvt.rn.f16x2.e4m3x2 %0, hi; }" : "=r"(y) : "r"(w));
    else
        asm("{ .reg .b16 lo, hi; mov.b32 {lo, hi}, %1; cvt.rn.f16x2.e4m3x2 %0, lo; }" : "=r"(y) : "r"(w));
    return y;
}
__device__ __forceinline__ uint32_t codes_to_half2(uint32_t w, int pair, Int8) {
    // 0x6400 + u is 1024 + u in fp16 for a byte u = code + 128
    const uint32_t u = __byte_perm(w ^ 0x80808080u, 0x64646464u, pair ? 0x4342 : 0x4140);
    const uint32_t bias = 0x64806480u;    // 1024 + 128
    const __half2 x = __hsub2(*reinterpret_cast<const __half2 *>(&u), *reinterpret_cast<const __half2 *>(&bias));
    return *reinterpret_cast<const uint32_t *>(&x);
}
