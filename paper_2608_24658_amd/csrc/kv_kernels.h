/*
 * kv_kernels.h -- the paged cache's write and read for gfx950.
 *
 * Both move every value once: a group of lanes takes one head of one token, of
 * keys or of values, eight values a lane.  The write needs the head's largest
 * magnitude before its first code, which the group finds by exchanges among
 * its lanes, so the values stay in registers between the two.  Bound by memory:
 * 182,000 positions of 8 heads of 128 values from FP8 pages of 24 slots to
 * bfloat16, 1.13 GB in all, take 256 us (4.4 TB/s, where a copy reaches 4.75);
 * 23,500 float16 tokens of 8 heads of 64 values to INT8 and back 44 us, two
 * launches of 74 MB each.  A single token of 64 rows is two launches and the
 * host's checks, 23 us.
 */
#pragma once
#include "kv_common.h"

namespace pk {

constexpr int KV_THREADS = 256;
constexpr int KV_PER_LANE = 8;  /* values */
/* Units of a lane on their way at once: a unit's page is a load that its values wait for, so one at a time leaves the
 * memory idle.  48 rows of 1 to 36,000 positions read from FP8: 390 us with one, 260 with these. */
constexpr int KV_WRITES = 2, KV_READS = 4;

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

/* A lane's eight values are two fours, at value lo and hi of the head: neighbours for 16-bit token arrays, 16 bytes in
 * all; for float32 ones half the group's lanes apart, so that neighbouring lanes read neighbouring 16 bytes. */
template <int T>
__device__ __forceinline__ int piece_lo(int lane) { return lane * (T == PARASON_DTYPE_F32 ? 4 : 8); }
template <int T>
__device__ __forceinline__ int piece_hi(int lane, int group) { return T == PARASON_DTYPE_F32 ? (group + lane) * 4 : lane * 8 + 4; }

/* T: type of the token arrays, PARASON_DTYPE_F32, _BF16 or _F16; p: the head */
template <int T>
__device__ __forceinline__ void load8(const char *p, int lo, int hi, bool hi_live, bool wide, float *x)
{
    if (T == PARASON_DTYPE_F32) {
        const float *f = reinterpret_cast<const float *>(p);
        if (wide) {
            float4 a = *reinterpret_cast<const float4 *>(f + lo), b = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
            if (hi_live) b = *reinterpret_cast<const float4 *>(f + hi);
            x[0] = a.x, x[1] = a.y, x[2] = a.z, x[3] = a.w, x[4] = b.x, x[5] = b.y, x[6] = b.z, x[7] = b.w;
        } else {
            for (int e = 0; e < 4; ++e) x[e] = f[lo + e];
            for (int e = 0; e < 4; ++e) x[4 + e] = hi_live ? f[hi + e] : 0.0f;
        }
        return;
    }
    uint32_t h[8];
    if (wide) {
        const uint4 a = *reinterpret_cast<const uint4 *>(p + lo * 2);
        const uint32_t w[4] = {a.x, a.y, a.z, a.w};
        for (int e = 0; e < 8; ++e) h[e] = (w[e / 2] >> (16 * (e & 1))) & 0xFFFFu;
    } else {
        for (int e = 0; e < 8; ++e) h[e] = reinterpret_cast<const uint16_t *>(p)[lo + e];
    }
    for (int e = 0; e < 8; ++e) x[e] = T == PARASON_DTYPE_BF16 ? bf16_to_f32(h[e]) : f16_to_f32(h[e]);
}

template <bool F16>
__device__ __forceinline__ uint4 pack8(const float *x)
{
    uint32_t h[8];
    for (int e = 0; e < 8; ++e) h[e] = F16 ? f32_to_f16(x[e]) : f32_to_bf16(x[e]);
    return make_uint4(h[0] | (h[1] << 16), h[2] | (h[3] << 16), h[4] | (h[5] << 16), h[6] | (h[7] << 16));
}

template <int T>
__device__ __forceinline__ void store8(char *p, int lo, int hi, bool hi_live, bool wide, const float *x)
{
    if (T == PARASON_DTYPE_F32) {
        float *f = reinterpret_cast<float *>(p);
        if (wide) {
            *reinterpret_cast<float4 *>(f + lo) = make_float4(x[0], x[1], x[2], x[3]);
            if (hi_live) *reinterpret_cast<float4 *>(f + hi) = make_float4(x[4], x[5], x[6], x[7]);
        } else {
            for (int e = 0; e < 4; ++e) f[lo + e] = x[e];
            for (int e = 0; e < 4; ++e)
                if (hi_live) f[hi + e] = x[4 + e];
        }
        return;
    }
    const uint4 r = pack8<T == PARASON_DTYPE_F16>(x);
    if (wide) {
        *reinterpret_cast<uint4 *>(p + lo * 2) = r;
    } else {
        const uint32_t w[4] = {r.x, r.y, r.z, r.w};
        for (int e = 0; e < 8; ++e) reinterpret_cast<uint16_t *>(p)[lo + e] = (uint16_t)(w[e / 2] >> (16 * (e & 1)));
    }
}

template <int T>
constexpr int type_bytes() { return T == PARASON_DTYPE_F32 ? 4 : 2; }

/* Where unit u of a row (token, k or v, head; head fastest) is. */
struct KvUnit {
    int32_t page, slot, head, token;
    bool is_v;
};

__device__ __forceinline__ KvUnit kv_unit(const KvMoveArgs &a, int64_t row, const KvRow &w, int64_t u, int64_t units)
{
    KvUnit x;
    const uint32_t v = (uint32_t)(u < units ? u : units - 1);
    const uint32_t th = div_by(v, a.heads_div); /* token * 2 + (k or v) */
    x.head = (int32_t)(v - th * (uint32_t)a.c.n_heads);
    x.token = (int32_t)(th >> 1);
    x.is_v = th & 1;
    x.page = page_of(a.r, a.c, row, w.kv_len - w.length + x.token, &x.slot);
    return x;
}

/* Blocks blocks_per_row * i .. take the units of row i in turn, KV_WRITES (KV_READS)
 * steps of a block at a time, so that this many pages and then this many
 * pieces of every lane are on their way at once. */
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
    const int64_t step = KV_THREADS >> a.group_log, units = (int64_t)w.length * 2 * a.c.n_heads;
    const int lo = piece_lo<T>(lane), hi = piece_hi<T>(lane, a.group);
    const bool live = lo < a.c.head_dim, hi_live = hi < a.c.head_dim;
    for (int64_t u0 = part * step * KV_WRITES; u0 < units; u0 += a.blocks_per_row * step * KV_WRITES) {
        KvUnit x[KV_WRITES];
        float f[KV_WRITES][8];
        bool mine[KV_WRITES];
#pragma unroll
        for (int i = 0; i < KV_WRITES; ++i) x[i] = kv_unit(a, row, w, u0 + i * step + (threadIdx.x >> a.group_log), units);
#pragma unroll
        for (int i = 0; i < KV_WRITES; ++i) {
            const bool there = u0 + i * step + (threadIdx.x >> a.group_log) < units;
            if (there && x[i].page < 0 && lane == 0) report(a.r, row, PARASON_KV_BAD_PAGE);
            mine[i] = there && live && x[i].page >= 0;
#pragma unroll
            for (int e = 0; e < 8; ++e) f[i][e] = 0.0f;
            if (mine[i])
                load8<T>((x[i].is_v ? a.v : a.k) + ((w.start + x[i].token) * a.stride_token + x[i].head * a.stride_head) *
                                                       type_bytes<T>(),
                         lo, hi, hi_live, a.wide, f[i]);
        }
#pragma unroll
        for (int i = 0; i < KV_WRITES; ++i) {
            char *cache = x[i].is_v ? a.c.v : a.c.k;
            const int64_t at = (int64_t)x[i].page * a.c.stride_page + (int64_t)x[i].slot * a.c.stride_slot +
                               x[i].head * a.c.stride_head;
            if (!CODES) {
                if (mine[i]) {
                    const uint4 p = pack8<KIND == KV_F16>(f[i]);
                    if (T == PARASON_DTYPE_F32) {
                        *reinterpret_cast<uint2 *>(cache + (at + lo) * 2) = make_uint2(p.x, p.y);
                        if (hi_live) *reinterpret_cast<uint2 *>(cache + (at + hi) * 2) = make_uint2(p.z, p.w);
                    } else {
                        *reinterpret_cast<uint4 *>(cache + (at + lo) * 2) = p;
                    }
                }
                continue;
            }
            /* the largest magnitude as bits: in that order infinities and NaN come last */
            uint32_t top = 0;
#pragma unroll
            for (int e = 0; e < 8; ++e) top = max(top, __float_as_uint(f[i][e]) & 0x7FFFFFFFu);
            for (int o = a.group >> 1; o > 0; o >>= 1) top = max(top, (uint32_t)__shfl_xor((int)top, o));
            const bool finite = top < 0x7F800000u;
            float scale = fmaxf(__uint_as_float(top) * (KIND == KV_FP8 ? 1.0f / 448.0f : 1.0f / 127.0f), 0x1p-126f);
            if (!finite) scale = __uint_as_float(0x7FC00000u);
#pragma unroll
            for (int e = 0; e < 8; ++e) f[i][e] = finite ? f[i][e] / scale : 0.0f;
            if (!mine[i]) continue;
            const uint2 codes = KIND == KV_FP8 ? make_uint2(f32_to_fp8x4(f[i]), f32_to_fp8x4(f[i] + 4))
                                               : make_uint2(f32_to_int8x4(f[i]), f32_to_int8x4(f[i] + 4));
            if (T == PARASON_DTYPE_F32) {
                *reinterpret_cast<uint32_t *>(cache + at + lo) = codes.x;
                if (hi_live) *reinterpret_cast<uint32_t *>(cache + at + hi) = codes.y;
            } else {
                *reinterpret_cast<uint2 *>(cache + at + lo) = codes;
            }
            if (lane == 0)
                (x[i].is_v ? a.c.v_scale : a.c.k_scale)[(int64_t)x[i].page * a.c.scale_stride_page +
                                                        (int64_t)x[i].slot * a.c.scale_stride_slot +
                                                        x[i].head * a.c.scale_stride_head] = scale;
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
    const int64_t step = KV_THREADS >> a.group_log, units = (int64_t)w.length * 2 * a.c.n_heads;
    const int lo = piece_lo<T>(lane), hi = piece_hi<T>(lane, a.group);
    if (lo >= a.c.head_dim) return;
    const bool hi_live = hi < a.c.head_dim;
    for (int64_t u0 = part * step * KV_READS; u0 < units; u0 += a.blocks_per_row * step * KV_READS) {
        KvUnit x[KV_READS];
        uint4 raw[KV_READS];
        float scale[KV_READS];
#pragma unroll
        for (int i = 0; i < KV_READS; ++i) x[i] = kv_unit(a, row, w, u0 + i * step + (threadIdx.x >> a.group_log), units);
#pragma unroll
        for (int i = 0; i < KV_READS; ++i) {
            raw[i] = make_uint4(0u, 0u, 0u, 0u);
            scale[i] = __uint_as_float(0x7FC00000u);
            if (x[i].page < 0) {
                if (lane == 0) report(a.r, row, PARASON_KV_BAD_PAGE);
                continue;
            }
            const char *cache = x[i].is_v ? a.c.v : a.c.k;
            const int64_t at = (int64_t)x[i].page * a.c.stride_page + (int64_t)x[i].slot * a.c.stride_slot +
                               x[i].head * a.c.stride_head;
            const int other = hi_live ? hi : lo;
            if (!CODES) {
                if (T == PARASON_DTYPE_F32) {
                    const uint2 p = *reinterpret_cast<const uint2 *>(cache + (at + lo) * 2);
                    const uint2 q = *reinterpret_cast<const uint2 *>(cache + (at + other) * 2);
                    raw[i] = make_uint4(p.x, p.y, q.x, q.y);
                } else {
                    raw[i] = *reinterpret_cast<const uint4 *>(cache + (at + lo) * 2);
                }
                scale[i] = 1.0f;
            } else {
                if (T == PARASON_DTYPE_F32) {
                    raw[i].x = *reinterpret_cast<const uint32_t *>(cache + at + lo);
                    raw[i].y = *reinterpret_cast<const uint32_t *>(cache + at + other);
                } else {
                    const uint2 codes = *reinterpret_cast<const uint2 *>(cache + at + lo);
                    raw[i].x = codes.x, raw[i].y = codes.y;
                }
                scale[i] = (x[i].is_v ? a.c.v_scale : a.c.k_scale)[(int64_t)x[i].page * a.c.scale_stride_page +
                                                                   (int64_t)x[i].slot * a.c.scale_stride_slot +
                                                                   x[i].head * a.c.scale_stride_head];
            }
        }
#pragma unroll
        for (int i = 0; i < KV_READS; ++i) {
            if (u0 + i * step + (threadIdx.x >> a.group_log) >= units) continue;
            float f[8];
            if (!CODES) {
                const uint32_t h[4] = {raw[i].x, raw[i].y, raw[i].z, raw[i].w};
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const uint32_t b = (h[e / 2] >> (16 * (e & 1))) & 0xFFFFu;
                    f[e] = x[i].page < 0 ? scale[i] : KIND == KV_BF16 ? bf16_to_f32(b) : f16_to_f32(b);
                }
            } else {
                if (KIND == KV_FP8) fp8x4_to_f32(raw[i].x, f), fp8x4_to_f32(raw[i].y, f + 4);
                else int8x4_to_f32(raw[i].x, f), int8x4_to_f32(raw[i].y, f + 4);
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    f[e] *= scale[i];
                    /* the product is a float: not one with the rounding to float16 behind it */
                    if (T == PARASON_DTYPE_F16) asm("" : "+v"(f[e]));
                }
            }
            store8<T>((x[i].is_v ? a.v : a.k) + ((w.start + x[i].token) * a.stride_token + x[i].head * a.stride_head) * type_bytes<T>(),
                      lo, hi, hi_live, a.wide, f);
        }
    }
}

/* ---- 4-bit caches ---------------------------------------------------------
 * A lane has eight values, and four lanes share a scale.  So little a head and
 * lane that finding its place and waiting for its page is most of the work: a
 * group takes HEADS heads of a token's keys or values, whose places are one
 * stride apart, and where these are fewer than four, several tokens at a time.
 * 182,000 positions of 8 heads of 128 values read as bfloat16, 0.94 GB, take 204
 * us with 8 heads, 222 with 4 and 266 with one (and four tokens); the tokens of
 * 64 rows, where there are too few groups otherwise, 5.0 with 8 and 3.9 with 4.
 * 256,000 tokens of one head of 128 values: written in 46 us four at a time,
 * read in 38; 63 and 49 one by one. */
constexpr int KV4_HEADS = 4, KV4_MORE = 8;
/* Tokens that are read KV4_MORE heads at a time.  Fewer leave too few groups, 2,048 of 8 heads of 128 values as bfloat16
 * 5.3 us and 4.5 with four heads; from here on the two are within 3 % of each other or eight are faster, 131,072 tokens of
 * 5 heads of 64 values 27.1 and 33.0 us, of 8 heads of 128 133.8 and 136.5 (float32 results up to 6 % either way). */
constexpr int64_t KV4_MANY = 16384;

struct Kv4Unit {
    int32_t page, token, head, heads; /* its first head, and how many (0: no unit) */
    bool is_v;
    char *codes;                      /* of the first head */
    uint8_t *scales;
};

/* Unit u of a row (token, k or v, HEADS heads; these fastest). */
template <int HEADS>
__device__ __forceinline__ Kv4Unit kv4_unit(const KvMoveArgs &a, int64_t row, const KvRow &w, int64_t u, int64_t units)
{
    Kv4Unit x;
    const uint32_t v = (uint32_t)(u < units ? u : units - 1), th = div_by(v, a.heads_div);
    x.head = (int32_t)(v - th * a.heads_div.d) * HEADS;
    x.heads = u >= units ? 0 : a.c.n_heads - x.head < HEADS ? a.c.n_heads - x.head : HEADS;
    x.token = (int32_t)(th >> 1);
    x.is_v = th & 1;
    int32_t slot;
    x.page = page_of(a.r, a.c, row, w.kv_len - w.length + x.token, &slot);
    const int64_t page = x.page < 0 ? 0 : x.page;
    x.codes = (x.is_v ? a.c.v : a.c.k) + ((page * a.c.stride_page + slot * a.c.stride_slot + x.head * a.c.stride_head) >> 1);
    x.scales = reinterpret_cast<uint8_t *>(x.is_v ? a.c.v_scale : a.c.k_scale) +
               (page * a.c.scale_stride_page + slot * a.c.scale_stride_slot + x.head * a.c.scale_stride_head);
    return x;
}

template <int T, int HEADS>
__global__ void __launch_bounds__(KV_THREADS) kv_write4(KvMoveArgs a)
{
    const int64_t row = blockIdx.x / (uint32_t)a.blocks_per_row;
    const uint32_t part = blockIdx.x % (uint32_t)a.blocks_per_row;
    const KvRow w = load_row(a.r, a.c, row, true);
    if (!w.ok) {
        if (part == 0 && threadIdx.x == 0) report(a.r, row, PARASON_KV_BAD_ROW);
        return;
    }
    constexpr int TOKENS = HEADS < KV4_HEADS ? KV4_HEADS / HEADS : 1;
    const int lane = (int)threadIdx.x & (a.group - 1), lo = lane * KV_PER_LANE;
    const bool live = lo < a.c.head_dim;
    const int64_t step = KV_THREADS >> a.group_log, units = (int64_t)w.length * 2 * a.heads_div.d;
    for (int64_t u0 = part * step * TOKENS; u0 < units; u0 += a.blocks_per_row * step * TOKENS) {
        Kv4Unit x[TOKENS];
        float f[TOKENS][HEADS][8];
#pragma unroll
        for (int k = 0; k < TOKENS; ++k) x[k] = kv4_unit<HEADS>(a, row, w, u0 + k * step + (threadIdx.x >> a.group_log), units);
#pragma unroll
        for (int k = 0; k < TOKENS; ++k) {
            if (x[k].page < 0 && x[k].heads > 0 && lane == 0) report(a.r, row, PARASON_KV_BAD_PAGE);
            const char *from =
                (x[k].is_v ? a.v : a.k) + ((w.start + x[k].token) * a.stride_token + x[k].head * a.stride_head) * type_bytes<T>();
#pragma unroll
            for (int i = 0; i < HEADS; ++i) {
#pragma unroll
                for (int e = 0; e < 8; ++e) f[k][i][e] = 0.0f;
                if (live && x[k].page >= 0 && i < x[k].heads)
                    load8<T>(from + i * a.stride_head * type_bytes<T>(), lo, lo + 4, true, a.wide, f[k][i]);
            }
        }
#pragma unroll
        for (int k = 0; k < TOKENS; ++k)
#pragma unroll
            for (int i = 0; i < HEADS; ++i) {
                /* the largest magnitude as bits: in that order infinities and NaN come last */
                uint32_t top = 0;
#pragma unroll
                for (int e = 0; e < 8; ++e) top = max(top, __float_as_uint(f[k][i][e]) & 0x7FFFFFFFu);
                top = max(top, (uint32_t)__shfl_xor((int)top, 1));
                top = max(top, (uint32_t)__shfl_xor((int)top, 2));
                if (!live || x[k].page < 0 || i >= x[k].heads) continue;
                const bool finite = top < 0x7F800000u;
                const uint32_t byte = finite ? fp4_scale_byte(top) : 255u;
                *reinterpret_cast<uint32_t *>(x[k].codes + ((i * a.c.stride_head + lo) >> 1)) =
                    finite ? f32_to_fp4x8(f[k][i], fp4_scale(byte)) : 0u;
                if ((lane & 3) == 0) x[k].scales[i * a.c.scale_stride_head + lo / PARASON_KV_SCALE_GROUP] = (uint8_t)byte;
            }
    }
}

/* float32 results: a lane's two fours are half the head apart, so that neighbouring lanes write neighbouring 16 bytes
 * (64,000 tokens of 8 heads of 128 values 165 us, 213 with 32 bytes a lane). */
template <int T, int HEADS>
__global__ void __launch_bounds__(KV_THREADS) kv_read4(KvMoveArgs a)
{
    const int64_t row = blockIdx.x / (uint32_t)a.blocks_per_row;
    const uint32_t part = blockIdx.x % (uint32_t)a.blocks_per_row;
    const KvRow w = load_row(a.r, a.c, row, true);
    if (!w.ok) {
        if (part == 0 && threadIdx.x == 0) report(a.r, row, PARASON_KV_BAD_ROW);
        return;
    }
    constexpr int TOKENS = HEADS < KV4_HEADS ? KV4_HEADS / HEADS : 1;
    constexpr bool F32 = T == PARASON_DTYPE_F32;
    const int lane = (int)threadIdx.x & (a.group - 1);
    if (lane * KV_PER_LANE >= a.c.head_dim) return;
    const int lo = F32 ? lane * 4 : lane * 8, hi = F32 ? a.c.head_dim / 2 + lane * 4 : lo + 4;
    const int64_t step = KV_THREADS >> a.group_log, units = (int64_t)w.length * 2 * a.heads_div.d;
    for (int64_t u0 = part * step * TOKENS; u0 < units; u0 += a.blocks_per_row * step * TOKENS) {
        Kv4Unit x[TOKENS];
        uint32_t codes[TOKENS][HEADS], byte[TOKENS][HEADS], last[TOKENS][HEADS]; /* last: the second four's scale */
#pragma unroll
        for (int k = 0; k < TOKENS; ++k) x[k] = kv4_unit<HEADS>(a, row, w, u0 + k * step + (threadIdx.x >> a.group_log), units);
#pragma unroll
        for (int k = 0; k < TOKENS; ++k) {
#pragma unroll
            for (int i = 0; i < HEADS; ++i) {
                codes[k][i] = 0u, byte[k][i] = last[k][i] = 255u; /* (of a bad page: NaN) */
                if (x[k].page < 0 || i >= x[k].heads) continue;
                const char *c = x[k].codes + ((i * a.c.stride_head) >> 1);
                const uint8_t *s = x[k].scales + i * a.c.scale_stride_head;
                if (F32) {
                    codes[k][i] = *reinterpret_cast<const uint16_t *>(c + lo / 2) | (uint32_t) * reinterpret_cast<const uint16_t *>(c + hi / 2) << 16;
                    last[k][i] = s[hi / PARASON_KV_SCALE_GROUP];
                } else {
                    codes[k][i] = *reinterpret_cast<const uint32_t *>(c + lo / 2);
                }
                byte[k][i] = s[lo / PARASON_KV_SCALE_GROUP];
            }
            if (x[k].page < 0 && x[k].heads > 0 && lane == 0) report(a.r, row, PARASON_KV_BAD_PAGE);
        }
#pragma unroll
        for (int k = 0; k < TOKENS; ++k) {
            char *to = (x[k].is_v ? a.v : a.k) + ((w.start + x[k].token) * a.stride_token + x[k].head * a.stride_head) * type_bytes<T>();
#pragma unroll
            for (int i = 0; i < HEADS; ++i) {
                float f[8], g[8];
                fp4x8_to_f32(codes[k][i], fp4_scale(byte[k][i]), f);
                if (F32) {
                    fp4x8_to_f32(codes[k][i], fp4_scale(last[k][i]), g);
#pragma unroll
                    for (int e = 4; e < 8; ++e) f[e] = g[e];
                }
                if (i < x[k].heads) store8<T>(to + i * a.stride_head * type_bytes<T>(), lo, hi, true, a.wide, f);
            }
        }
    }
}

}  // namespace pk
