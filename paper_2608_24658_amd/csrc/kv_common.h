/*
 * kv_common.h -- what the cache's kernels and the attention that reads it
 * share: the device views of a cache and of a call's rows, a row's bounds,
 * the place of a position, and the 8- and 4-bit codes.
 */
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "parason.h"

namespace pk {

/* n / d for 0 <= n < 2^31 by a multiplication: with l = ceil(log2 d) and
 * m = floor(2^(31 + l) / d) + 1, n * m / 2^(31 + l) exceeds n / d by less than
 * n / 2^(31 + l) <= 2^-l <= 1 / d, too little to reach the next integer. */
struct FastDiv {
    uint32_t d, m, s;
};

inline FastDiv fast_div(uint32_t d)
{
    uint32_t l = 0;
    while ((1ull << l) < d) ++l;
    return FastDiv{d, (uint32_t)((1ull << (31 + l)) / d + 1), l};
}

__device__ __forceinline__ uint32_t div_by(uint32_t n, const FastDiv &f)
{
    return (uint32_t)(((uint64_t)n * f.m) >> (31 + f.s));
}

enum : int { KV_BF16 = 0, KV_F16, KV_FP8, KV_INT8, KV_FP4 };

/* Bytes of n values of a cache. */
template <int KIND>
__device__ __forceinline__ constexpr int64_t cache_bytes(int64_t n)
{
    return KIND == KV_FP4 ? n / 2 : KIND == KV_FP8 || KIND == KV_INT8 ? n : n * 2;
}

struct KvCache {
    char *k, *v;
    float *k_scale, *v_scale;                                        /* 4-bit caches: bytes */
    int64_t n_pages;
    int64_t stride_page, stride_slot, stride_head;                   /* elements */
    int64_t scale_stride_page, scale_stride_slot, scale_stride_head;
    int32_t page_size, n_heads, head_dim;
    FastDiv page_div;
};

struct KvRows {
    int64_t n_rows, n_tokens;
    const int64_t *starts;
    const int32_t *lengths, *kv_lens, *pages;
    int64_t pages_stride;
    int32_t max_pages, max_length, max_kv_len;
    uint32_t *status;
};

/* A row as the kernels take it.  `out_ok`: its tokens lie where the call's
 * arrays have room; `ok`: all of it can be evaluated. */
struct KvRow {
    int64_t start;
    int32_t length, kv_len;
    bool out_ok, ok;
};

__device__ __forceinline__ KvRow load_row(const KvRows &r, const KvCache &c, int64_t i, bool needs_positions)
{
    KvRow w;
    w.start = r.starts[i];
    w.length = r.lengths[i];
    w.kv_len = r.kv_lens[i];
    w.out_ok = w.length >= 0 && w.length <= r.max_length && w.start >= 0 && w.start <= r.n_tokens - w.length;
    w.ok = w.out_ok && w.kv_len >= 0 && w.kv_len <= r.max_kv_len &&
           (int64_t)w.kv_len <= (int64_t)r.max_pages * c.page_size && (!needs_positions || w.kv_len >= w.length);
    return w;
}

/* Page of position p of row i (-1: not a page of the cache), and its slot. */
__device__ __forceinline__ int32_t page_of(const KvRows &r, const KvCache &c, int64_t i, int32_t p, int32_t *slot)
{
    const uint32_t n = div_by((uint32_t)p, c.page_div);
    *slot = p - (int32_t)(n * (uint32_t)c.page_size);
    const int32_t page = r.pages[i * r.pages_stride + n];
    return page >= 0 && page < c.n_pages ? page : -1;
}

__device__ __forceinline__ void report(const KvRows &r, int64_t i, uint32_t bits)
{
    if (r.status) atomicOr(&r.status[i], bits);
}

/* ---- 16- and 8-bit values -------------------------------------------------- */

__device__ __forceinline__ float bf16_to_f32(uint32_t h) { return __uint_as_float(h << 16); }

/* Round to nearest even; NaN stays NaN. */
__device__ __forceinline__ uint32_t f32_to_bf16(float x)
{
    typedef __bf16 bf16;
    return (uint32_t)__builtin_bit_cast(uint16_t, (bf16)x);
}

__device__ __forceinline__ float f16_to_f32(uint32_t h) { return (float)__builtin_bit_cast(_Float16, (uint16_t)h); }

__device__ __forceinline__ uint32_t f32_to_f16(float x)
{
    return (uint32_t)__builtin_bit_cast(uint16_t, (_Float16)x);
}

/* Four codes of one 32-bit word as floats. */
__device__ __forceinline__ void fp8x4_to_f32(uint32_t w, float *x)
{
    typedef float f2 __attribute__((ext_vector_type(2)));
    const f2 a = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, false), b = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, true);
    x[0] = a.x, x[1] = a.y, x[2] = b.x, x[3] = b.y;
}

__device__ __forceinline__ void int8x4_to_f32(uint32_t w, float *x)
{
    x[0] = (float)(int8_t)w, x[1] = (float)(int8_t)(w >> 8), x[2] = (float)(int8_t)(w >> 16),
    x[3] = (float)(int8_t)(w >> 24);
}

/* Four values, |x| <= 448 (but for a rounding), to e4m3 codes. */
__device__ __forceinline__ uint32_t f32_to_fp8x4(const float *x)
{
    int w = __builtin_amdgcn_cvt_pk_fp8_f32(x[0], x[1], 0, false);
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(x[2], x[3], w, true);
}

__device__ __forceinline__ uint32_t f32_to_int8x4(const float *x)
{
    uint32_t w = 0;
#pragma unroll
    for (int e = 0; e < 4; ++e) w |= ((uint32_t)(int32_t)__builtin_rintf(x[e]) & 255u) << (8 * e);
    return w;
}

/* The power of two that 32 values of four bits share, as the conversions take
 * it: they read a float's exponent field, and 255 there (a byte of 255) makes
 * every value NaN. */
__device__ __forceinline__ float fp4_scale(uint32_t byte) { return __uint_as_float(byte << 23); }

/* Eight codes of one 32-bit word, times their power of two: exact. */
__device__ __forceinline__ void fp4x8_to_f32(uint32_t w, float scale, float *x)
{
    typedef float f2 __attribute__((ext_vector_type(2)));
    const f2 a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, scale, 0), b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, scale, 1);
    const f2 c = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, scale, 2), d = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, scale, 3);
    x[0] = a.x, x[1] = a.y, x[2] = b.x, x[3] = b.y, x[4] = c.x, x[5] = c.y, x[6] = d.x, x[7] = d.y;
}

/* Eight values to codes: divided by their power of two, rounded to nearest even, at most 6. */
__device__ __forceinline__ uint32_t f32_to_fp4x8(const float *x, float scale)
{
    uint32_t w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(0u, x[0], x[1], scale, 0);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[2], x[3], scale, 1);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[4], x[5], scale, 2);
    return __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[6], x[7], scale, 3);
}

/* The byte of the least power of two, within the bounds of parason.h, with amax
 * <= 7 times it; top: amax's bits, finite. */
__device__ __forceinline__ uint32_t fp4_scale_byte(uint32_t top)
{
    /* amax = f * 2^(E - 127), 1 <= f < 2: E - 2 for f <= 1.75, else E - 1 (the carry of the fraction) */
    const int32_t e = (int32_t)((top + 0x1FFFFFu) >> 23) - 2;
    return (uint32_t)(e < 7 ? 7 : e > 252 ? 252 : e);
}

}  // namespace pk
