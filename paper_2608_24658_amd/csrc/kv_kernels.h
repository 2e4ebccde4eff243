/*
 * kv_kernels.h -- the paged cache's write and read for gfx950.
 *
 * Both move every value once: a group of lanes takes one head of one token, of
 * keys or of values, eight values a lane.  The write needs the head's largest
 * magnitude before its first code, which the group finds by exchanges among
 * its lanes, so the values stay in registers between the two.  Bound by memory.
 */
#pragma once
#include "kv_common.h"

namespace pk {

constexpr int KV_THREADS = 256;
constexpr int KV_PER_LANE = 8;  /* values */

struct KvMoveArgs {
    KvCache c;
    KvRows r;
    char *k, *v;              /* the call's token arrays */
    int64_t stride_token, stride_head;
    int32_t group;            /* lanes per head: the power of two that holds head_dim / 8 */
    int32_t group_log;
    int32_t blocks_per_row;
    FastDiv heads_div;
    bool wide;                /* the token arrays are 16-byte aligned throughout */
};

/* type of the token arrays: PARASON_DTYPE_F32, _BF16, _F16 */
template <int T>
__device__ __forceinline__ void load8(const char *p, bool wide, float *x)
{
    if (T == PARASON_DTYPE_F32) {
        const float *f = reinterpret_cast<const float *>(p);
        if (wide) {
            const float4 a = reinterpret_cast<const float4 *>(p)[0], b = reinterpret_cast<const float4 *>(p)[1];
            x[0] = a.x, x[1] = a.y, x[2] = a.z, x[3] = a.w, x[4] = b.x, x[5] = b.y, x[6] = b.z, x[7] = b.w;
        } else {
            for (int e = 0; e < 8; ++e) x[e] = f[e];
        }
        return;
    }
    uint32_t h[8];
    if (wide) {
        const uint4 a = *reinterpret_cast<const uint4 *>(p);
        const uint32_t w[4] = {a.x, a.y, a.z, a.w};
        for (int e = 0; e < 8; ++e) h[e] = (w[e / 2] >> (16 * (e & 1))) & 0xFFFFu;
    } else {
        for (int e = 0; e < 8; ++e) h[e] = reinterpret_cast<const uint16_t *>(p)[e];
    }
    for (int e = 0; e < 8; ++e) x[e] = T == PARASON_DTYPE_BF16 ? bf16_to_f32(h[e]) : f16_to_f32(h[e]);
}

template <int T>
__device__ __forceinline__ void store8(char *p, bool wide, const float *x)
{
    if (T == PARASON_DTYPE_F32) {
        float *f = reinterpret_cast<float *>(p);
        if (wide) {
            reinterpret_cast<float4 *>(p)[0] = make_float4(x[0], x[1], x[2], x[3]);
            reinterpret_cast<float4 *>(p)[1] = make_float4(x[4], x[5], x[6], x[7]);
        } else {
            for (int e = 0; e < 8; ++e) f[e] = x[e];
        }
        return;
    }
    uint32_t h[8];
    for (int e = 0; e < 8; ++e) h[e] = T == PARASON_DTYPE_BF16 ? f32_to_bf16(x[e]) : f32_to_f16(x[e]);
    if (wide) {
        *reinterpret_cast<uint4 *>(p) =
            make_uint4(h[0] | (h[1] << 16), h[2] | (h[3] << 16), h[4] | (h[5] << 16), h[6] | (h[7] << 16));
    } else {
        for (int e = 0; e < 8; ++e) reinterpret_cast<uint16_t *>(p)[e] = (uint16_t)h[e];
    }
}

template <int T>
constexpr int type_bytes() { return T == PARASON_DTYPE_F32 ? 4 : 2; }

/* Blocks blocks_per_row * i .. take the heads of row i's tokens in turn: unit
 * (token, k or v, head), head fastest. */
template <int T, int KIND>
__global__ void __launch_bounds__(KV_THREADS) kv_write(KvMoveArgs a)
{
    const int64_t row = blockIdx.x / (uint32_t)a.blocks_per_row;
    const uint32_t part = blockIdx.x % (uint32_t)a.blocks_per_row;
    const KvRow w = load_row(a.r, a.c, row, true);
    if (!w.ok) {
        if (part == 0 && threadIdx.x == 0) report(a.r, row, PARASON_KV_BAD_ROW);
        return;
    }
    constexpr bool CODES = KIND == KV_FP8 || KIND == KV_INT8;
    const int lane = (int)threadIdx.x & (a.group - 1);
    const int per_block = KV_THREADS >> a.group_log;
    const int64_t units = (int64_t)w.length * 2 * a.c.n_heads;
    const int d0 = lane * KV_PER_LANE;
    const bool live = d0 < a.c.head_dim;
    for (int64_t u0 = (int64_t)part * per_block; u0 < units; u0 += (int64_t)a.blocks_per_row * per_block) {
        const int64_t u = u0 + (threadIdx.x >> a.group_log);
        const bool there = u < units; /* the same for the whole group of lanes */
        const uint32_t th = div_by((uint32_t)(there ? u : 0), a.heads_div); /* token * 2 + (k or v) */
        const int32_t head = (int32_t)((there ? u : 0) - (int64_t)th * a.c.n_heads);
        const int32_t j = (int32_t)(th >> 1);
        const bool is_v = th & 1;
        int32_t slot = 0, page = -1;
        if (there) {
            page = page_of(a.r, a.c, row, w.kv_len - w.length + j, &slot);
            if (page < 0 && lane == 0) report(a.r, row, PARASON_KV_BAD_PAGE);
        }
        const bool mine = live && page >= 0;
        float x[8] = {};
        if (mine)
            load8<T>((is_v ? a.v : a.k) +
                         ((w.start + j) * a.stride_token + head * a.stride_head + d0) * type_bytes<T>(),
                     a.wide, x);
        char *cache = is_v ? a.c.v : a.c.k;
        const int64_t at = (int64_t)page * a.c.stride_page + (int64_t)slot * a.c.stride_slot +
                           head * a.c.stride_head + d0;
        if (!CODES) {
            if (mine) store8<KIND == KV_BF16 ? PARASON_DTYPE_BF16 : PARASON_DTYPE_F16>(cache + at * 2, true, x);
            continue;
        }
        /* the largest magnitude as bits: in that order infinities and NaN come last */
        uint32_t top = 0;
        for (int e = 0; e < 8; ++e) top = max(top, __float_as_uint(x[e]) & 0x7FFFFFFFu);
        for (int o = a.group >> 1; o > 0; o >>= 1) top = max(top, (uint32_t)__shfl_xor((int)top, o));
        const bool finite = top < 0x7F800000u;
        float scale = fmaxf(__uint_as_float(top) * (KIND == KV_FP8 ? 1.0f / 448.0f : 1.0f / 127.0f), 0x1p-126f);
        if (!finite) scale = __uint_as_float(0x7FC00000u);
        for (int e = 0; e < 8; ++e) x[e] = finite ? x[e] / scale : 0.0f;
        if (mine) {
            const uint2 codes = KIND == KV_FP8 ? make_uint2(f32_to_fp8x4(x), f32_to_fp8x4(x + 4))
                                               : make_uint2(f32_to_int8x4(x), f32_to_int8x4(x + 4));
            *reinterpret_cast<uint2 *>(cache + at) = codes;
            if (lane == 0)
                (is_v ? a.c.v_scale : a.c.k_scale)[(int64_t)page * a.c.scale_stride_page +
                                                   (int64_t)slot * a.c.scale_stride_slot +
                                                   head * a.c.scale_stride_head] = scale;
        }
    }
}

template <int T, int KIND>
__global__ void __launch_bounds__(KV_THREADS) kv_read(KvMoveArgs a)
{
    const int64_t row = blockIdx.x / (uint32_t)a.blocks_per_row;
    const uint32_t part = blockIdx.x % (uint32_t)a.blocks_per_row;
    const KvRow w = load_row(a.r, a.c, row, true);
    if (!w.ok) {
        if (part == 0 && threadIdx.x == 0) report(a.r, row, PARASON_KV_BAD_ROW);
        return;
    }
    constexpr bool CODES = KIND == KV_FP8 || KIND == KV_INT8;
    const int lane = (int)threadIdx.x & (a.group - 1);
    const int per_block = KV_THREADS >> a.group_log;
    const int64_t units = (int64_t)w.length * 2 * a.c.n_heads;
    const int d0 = lane * KV_PER_LANE;
    if (d0 >= a.c.head_dim) return;
    for (int64_t u = (int64_t)part * per_block + (threadIdx.x >> a.group_log); u < units;
         u += (int64_t)a.blocks_per_row * per_block) {
        const uint32_t th = div_by((uint32_t)u, a.heads_div);
        const int32_t head = (int32_t)(u - (int64_t)th * a.c.n_heads);
        const int32_t j = (int32_t)(th >> 1);
        const bool is_v = th & 1;
        int32_t slot;
        const int32_t page = page_of(a.r, a.c, row, w.kv_len - w.length + j, &slot);
        float x[8];
        if (page < 0) {
            if (lane == 0) report(a.r, row, PARASON_KV_BAD_PAGE);
            for (int e = 0; e < 8; ++e) x[e] = __uint_as_float(0x7FC00000u);
        } else {
            const char *cache = is_v ? a.c.v : a.c.k;
            const int64_t at = (int64_t)page * a.c.stride_page + (int64_t)slot * a.c.stride_slot +
                               head * a.c.stride_head + d0;
            if (!CODES) {
                load8<KIND == KV_BF16 ? PARASON_DTYPE_BF16 : PARASON_DTYPE_F16>(cache + at * 2, true, x);
            } else {
                const uint2 codes = *reinterpret_cast<const uint2 *>(cache + at);
                const float scale = (is_v ? a.c.v_scale : a.c.k_scale)[(int64_t)page * a.c.scale_stride_page +
                                                                       (int64_t)slot * a.c.scale_stride_slot +
                                                                       head * a.c.scale_stride_head];
                if (KIND == KV_FP8) fp8x4_to_f32(codes.x, x), fp8x4_to_f32(codes.y, x + 4);
                else int8x4_to_f32(codes.x, x), int8x4_to_f32(codes.y, x + 4);
                for (int e = 0; e < 8; ++e) x[e] *= scale;
            }
        }
        store8<T>((is_v ? a.v : a.k) + ((w.start + j) * a.stride_token + head * a.stride_head + d0) * type_bytes<T>(),
                  a.wide, x);
    }
}

}  // namespace pk
