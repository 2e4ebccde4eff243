/*
 * rotate_kernels.h -- norm and rotation of query and key heads for gfx950, and
 * its backward pass.
 *
 * A group of lanes takes one head of one token, 16 values a lane as two pieces
 * of eight: the two halves of its pairs (or eight neighbouring pairs), so that a
 * lane rotates what it holds and only the sum of squares (backward: and the sum
 * that takes the norm's share out of the gradient) crosses lanes.  All heads of
 * a token turn by the same angles: a block takes a few tokens, whose sines and
 * cosines it works out once, and then all their heads.  Bound by memory: each
 * value is read once and written once (backward: read twice, written once).
 */
#pragma once
#include "kv_kernels.h"

namespace pk {

constexpr int ROT_THREADS = 256;
constexpr int ROT_TOKENS = 8;        /* most tokens of a block at a time */
constexpr int ROT_TURNS = 256;       /* most sines and cosines of these; one token has at most 128 */
constexpr int ROT_GRAD_BLOCKS = 1024; /* most blocks of the backward pass, each with a share of the weights' gradients */

struct RotHeads {
    char *q, *k;
    int64_t q_token, q_head, k_token, k_head; /* elements */
    bool wide;                   /* 16-byte aligned throughout */
};

struct RotArgs {
    RotHeads x, g, y;            /* g: the backward pass's gradient of the results */
    int64_t n_tokens;
    int32_t q_heads, k_heads, dim, half; /* half: pairs that are rotated */
    int32_t group_log, at_once;  /* lanes of a head (a power of two >= dim / 16); tokens of a block at a time */
    FastDiv q_div, k_div;        /* by the heads */
    float eps, inv_dim;
    const int32_t *positions;
    const double *freqs;
    const char *q_weight, *k_weight;
    float *sums;                 /* [blocks][2][dim] */
};

template <int T>
__device__ __forceinline__ void rot_load(const char *head, int at, bool wide, float *x)
{
    const char *p = head + at * type_bytes<T>();
    if (T == PARASON_DTYPE_F32) {
        load8<T>(p, 0, 4, true, wide, x);
    } else {
        load8<T>(p, 0, 0, true, wide, x);
    }
}

template <int T>
__device__ __forceinline__ void rot_store(char *head, int at, bool wide, const float *x)
{
    char *p = head + at * type_bytes<T>();
    if (T == PARASON_DTYPE_F32) {
        store8<T>(p, 0, 4, true, wide, x);
    } else {
        store8<T>(p, 0, 0, true, wide, x);
    }
}

/* cos and sin of position * freq.  The angle is reduced to half turns in [-1, 1]
 * in double and goes on as two floats, so that the float functions see all of
 * it: the second, below 2^-25, turns what the first gave by its own small angle. */
__device__ __forceinline__ float2 turn_of(int32_t position, double freq)
{
    double t = (double)position * freq * 0.15915494309189535;
    t = 2.0 * (t - __builtin_rint(t));
    const float hi = (float)t, lo = (float)(t - (double)hi) * 3.14159265358979f;
    float s, c;
    sincospif(hi, &s, &c);
    return make_float2(__builtin_fmaf(-s, lo, c), __builtin_fmaf(c, lo, s));
}

struct RotLds {
    float2 turns[ROT_TURNS];
    float w[2][PARASON_KV_MAX_DIM];
};

template <int T>
__device__ __forceinline__ void rot_weights(const RotArgs &a, RotLds &s)
{
    for (int i = (int)threadIdx.x; i < 2 * a.dim; i += ROT_THREADS) {
        const int which = i >= a.dim, d = i - which * a.dim;
        const char *w = which ? a.k_weight : a.q_weight;
        float x = 1.0f;
        if (w) {
            if (T == PARASON_DTYPE_F32) x = reinterpret_cast<const float *>(w)[d];
            else if (T == PARASON_DTYPE_BF16) x = bf16_to_f32(reinterpret_cast<const uint16_t *>(w)[d]);
            else x = f16_to_f32(reinterpret_cast<const uint16_t *>(w)[d]);
        }
        s.w[which][d] = x;
    }
}

/* The turns of tokens t0 .. t0 + n - 1. */
__device__ __forceinline__ void rot_turns(const RotArgs &a, RotLds &s, int64_t t0, int n)
{
    for (int i = (int)threadIdx.x; i < n * a.half; i += ROT_THREADS) {
        const int token = i / a.half, j = i - token * a.half;
        s.turns[i] = turn_of(a.positions[t0 + token], a.freqs[j]);
    }
}

/* A lane's two pieces of a head: values [lo, lo + 8) and [hi, hi + 8), pair e of
 * its eight being values e of both, or 2e and 2e + 1 of the 16. */
template <bool INTER>
struct RotPiece {
    int lo, hi;
    bool live, turned;

    __device__ __forceinline__ RotPiece(const RotArgs &a, int lane)
    {
        turned = lane * 8 < a.half;
        live = lane * 16 < a.dim;
        if (INTER || !turned) lo = lane * 16, hi = lo + 8;
        else lo = lane * 8, hi = a.half + lane * 8;
    }
};

/* x: 16 values; DIRECTION 1: by the angles, -1: back */
template <bool INTER, int DIRECTION>
__device__ __forceinline__ void rot_turn(float *x, const float2 *turns)
{
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const float2 cs = turns[e];
        const float s = DIRECTION > 0 ? cs.y : -cs.y;
        float &a = x[INTER ? 2 * e : e], &b = x[INTER ? 2 * e + 1 : 8 + e];
        const float na = __builtin_fmaf(a, cs.x, -(b * s)), nb = __builtin_fmaf(b, cs.x, a * s);
        a = na, b = nb;
    }
}

/* Unit u of a block's tokens: query heads first, then key heads. */
struct RotUnit {
    int token, head;
    bool is_k;
};

__device__ __forceinline__ RotUnit rot_unit(const RotArgs &a, int u, int q_units)
{
    RotUnit x;
    x.is_k = u >= q_units;
    const uint32_t v = (uint32_t)(x.is_k ? u - q_units : u);
    x.token = (int)div_by(v, x.is_k ? a.k_div : a.q_div);
    x.head = (int)v - x.token * (x.is_k ? a.k_heads : a.q_heads);
    return x;
}

template <int T>
__device__ __forceinline__ char *rot_head(const RotHeads &x, const RotUnit &u, int64_t t)
{
    const int64_t at = u.is_k ? t * x.k_token + u.head * x.k_head : t * x.q_token + u.head * x.q_head;
    return (u.is_k ? x.k : x.q) + at * type_bytes<T>();
}

__device__ __forceinline__ float group_sum(float x, int group_log)
{
    for (int k = 1; k < 1 << group_log; k <<= 1) x += __shfl_xor(x, k);
    return x;
}

template <int T, bool INTER>
__global__ void __launch_bounds__(ROT_THREADS) qk_norm_rotate(RotArgs a)
{
    __shared__ RotLds s;
    const int64_t t0 = (int64_t)blockIdx.x * a.at_once;
    const int n = (int)(a.n_tokens - t0 < a.at_once ? a.n_tokens - t0 : a.at_once);
    rot_weights<T>(a, s);
    rot_turns(a, s, t0, n);
    __syncthreads();
    const int lane = (int)threadIdx.x & ((1 << a.group_log) - 1);
    const RotPiece<INTER> p(a, lane);
    const int q_units = n * a.q_heads, units = q_units + n * a.k_heads, step = ROT_THREADS >> a.group_log;
    for (int u = (int)threadIdx.x >> a.group_log; u < units; u += step) {
        const RotUnit v = rot_unit(a, u, q_units);
        const int64_t t = t0 + v.token;
        float x[16] = {};
        if (p.live) {
            const char *h = rot_head<T>(a.x, v, t);
            rot_load<T>(h, p.lo, a.x.wide, x);
            rot_load<T>(h, p.hi, a.x.wide, x + 8);
        }
        float sum = 0.0f;
#pragma unroll
        for (int e = 0; e < 16; ++e) sum = __builtin_fmaf(x[e], x[e], sum);
        const float r = rsqrtf(__builtin_fmaf(group_sum(sum, a.group_log), a.inv_dim, a.eps));
        if (!p.live) continue;
        const float *w = s.w[v.is_k];
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] *= r * w[p.lo + e], x[8 + e] *= r * w[p.hi + e];
        if (p.turned) rot_turn<INTER, 1>(x, s.turns + v.token * a.half + lane * 8);
        if (a.positions[t] < 0) {
#pragma unroll
            for (int e = 0; e < 16; ++e) x[e] = 0.0f;
        }
        char *y = rot_head<T>(a.y, v, t);
        rot_store<T>(y, p.lo, a.y.wide, x);
        rot_store<T>(y, p.hi, a.y.wide, x + 8);
    }
}

/* The same with the gradient turned back; a lane always has the same values of
 * its heads and keeps its sums of the weights' gradients in registers.  The
 * block's groups of lanes are added at the end, in their order. */
template <int T, bool INTER>
__global__ void __launch_bounds__(ROT_THREADS) qk_norm_rotate_grad(RotArgs a)
{
    __shared__ RotLds s;
    __shared__ float sums[ROT_THREADS * 16];
    const int lane = (int)threadIdx.x & ((1 << a.group_log) - 1), groups = ROT_THREADS >> a.group_log;
    const int mine = (int)threadIdx.x >> a.group_log;
    const RotPiece<INTER> p(a, lane);
    float acc[2][16] = {};
    rot_weights<T>(a, s);
    for (int64_t t0 = (int64_t)blockIdx.x * a.at_once; t0 < a.n_tokens; t0 += (int64_t)gridDim.x * a.at_once) {
        const int n = (int)(a.n_tokens - t0 < a.at_once ? a.n_tokens - t0 : a.at_once);
        __syncthreads();
        rot_turns(a, s, t0, n);
        __syncthreads();
        const int q_units = n * a.q_heads, units = q_units + n * a.k_heads;
        for (int u = mine; u < units; u += groups) {
            const RotUnit v = rot_unit(a, u, q_units);
            const int64_t t = t0 + v.token;
            const bool there = a.positions[t] >= 0;
            float x[16] = {}, g[16] = {};
            if (p.live && there) {
                const char *h = rot_head<T>(a.x, v, t), *d = rot_head<T>(a.g, v, t);
                rot_load<T>(h, p.lo, a.x.wide, x);
                rot_load<T>(h, p.hi, a.x.wide, x + 8);
                rot_load<T>(d, p.lo, a.g.wide, g);
                rot_load<T>(d, p.hi, a.g.wide, g + 8);
                if (p.turned) rot_turn<INTER, -1>(g, s.turns + v.token * a.half + lane * 8);
            }
            const float *w = s.w[v.is_k];
            float sum = 0.0f, dot = 0.0f, gw[16];
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                gw[e] = g[e] * w[e < 8 ? p.lo + e : p.hi + e - 8];
                sum = __builtin_fmaf(x[e], x[e], sum);
                dot = __builtin_fmaf(gw[e], x[e], dot);
            }
            const float r = rsqrtf(__builtin_fmaf(group_sum(sum, a.group_log), a.inv_dim, a.eps));
            dot = group_sum(dot, a.group_log) * r * a.inv_dim;
            if (!p.live) continue;
#pragma unroll
            for (int e = 0; e < 16; ++e) x[e] *= r;
            if (v.is_k) {
#pragma unroll
                for (int e = 0; e < 16; ++e) acc[1][e] = __builtin_fmaf(g[e], x[e], acc[1][e]);
            } else {
#pragma unroll
                for (int e = 0; e < 16; ++e) acc[0][e] = __builtin_fmaf(g[e], x[e], acc[0][e]);
            }
#pragma unroll
            for (int e = 0; e < 16; ++e) x[e] = r * __builtin_fmaf(-x[e], dot, gw[e]);
            char *y = rot_head<T>(a.y, v, t);
            rot_store<T>(y, p.lo, a.y.wide, x);
            rot_store<T>(y, p.hi, a.y.wide, x + 8);
        }
    }
#pragma unroll
    for (int which = 0; which < 2; ++which) {
        __syncthreads();
        if (p.live) {
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                sums[mine * a.dim + p.lo + e] = acc[which][e];
                sums[mine * a.dim + p.hi + e] = acc[which][8 + e];
            }
        }
        __syncthreads();
        for (int d = (int)threadIdx.x; d < a.dim; d += ROT_THREADS) {
            float x = 0.0f;
            for (int i = 0; i < groups; ++i) x += sums[i * a.dim + d];
            a.sums[((int64_t)blockIdx.x * 2 + which) * a.dim + d] = x;
        }
    }
}

/* The blocks' sums of 16 values a block, 16 shares of them each, in double. */
__global__ void __launch_bounds__(ROT_THREADS) rotate_weight_grad(const float *sums, int32_t blocks, int32_t dim, float *q, float *k)
{
    __shared__ double part[16][17];
    const int col = (int)threadIdx.x & 15, share = (int)threadIdx.x >> 4;
    const int i = (int)blockIdx.x * 16 + col; /* of 2 * dim */
    double x = 0.0;
#pragma unroll 8
    for (int b = share; b < blocks; b += 16) x += (double)sums[(int64_t)b * 2 * dim + i];
    part[share][col] = x;
    __syncthreads();
    if (share != 0) return;
    x = 0.0;
    for (int b = 0; b < 16; ++b) x += part[b][col];
    float *to = i < dim ? q : k;
    if (to) to[i < dim ? i : i - dim] = (float)x;
}

}  // namespace pk
