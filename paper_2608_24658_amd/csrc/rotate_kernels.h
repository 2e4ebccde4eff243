/*
 * rotate_kernels.h -- norm and rotation of query and key heads for gfx950, and
 * its backward pass.
 *
 * A group of lanes takes one head of one token, 16 values a lane, eight pairs or
 * what is not rotated, so that a lane rotates what it holds and only the sum of
 * squares (backward: and the sum that takes the norm's share out of the
 * gradient) crosses lanes.  All heads of a token turn by the same angles: a
 * block takes a few tokens, whose sines and cosines it works out once, and then
 * all their heads.  Bound by memory: each value is read once and written once
 * (backward: read twice, written once).
 */
#pragma once
#include "kv_kernels.h"

namespace pk {

constexpr int ROT_THREADS = 256;
constexpr int ROT_TOKENS = 16;       /* most tokens of a block at a time */
constexpr int ROT_TURNS = 1024;      /* most sines and cosines of these; one token has at most 128 */
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

/* cos and sin of position * freq.  The product and its share of a turn are held
 * as two doubles each, so that what is left of many turns is exact too: a double
 * alone is off by 2^-53 of the whole angle, 2^-22 radians at 2^31.  The angle,
 * in half turns in [-1, 1], goes on as two floats, so that the float functions
 * see all of it: the second, below 2^-25, turns what the first gave by its own
 * small angle. */
__device__ __forceinline__ float2 turn_of(int32_t position, double freq)
{
    constexpr double PER_TURN = 0.15915494309189535, PER_TURN_LO = -9.839338337591243e-18; /* 1 / (2 pi) */
    const double p = (double)position, x = p * freq, x_lo = __builtin_fma(p, freq, -x);
    const double n = x * PER_TURN, n_lo = __builtin_fma(x, PER_TURN, -n) + __builtin_fma(x, PER_TURN_LO, x_lo * PER_TURN);
    const double t = 2.0 * ((n - __builtin_rint(n)) + n_lo);
    const float hi = (float)t, lo = (float)(t - (double)hi) * 3.14159265358979f;
    float s, c;
    sincospif(hi, &s, &c);
    return make_float2(__builtin_fmaf(-s, lo, c), __builtin_fmaf(c, lo, s));
}

struct RotLds {
    __attribute__((aligned(16))) float2 turns[ROT_TURNS];
    __attribute__((aligned(16))) float w[2][PARASON_KV_MAX_DIM];
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

/* A lane's 16 values of a head: four fours, at values q[0] .. q[3].  Neighbouring lanes have neighbouring 16 bytes (two
 * fours of a 16-bit type), so that every access of a group is whole lines (with 32 bytes of float32 a lane, 16 at a time,
 * 16,000 tokens of 14 heads of 80 values took 81 us forward, this 31).  Halves: pair e of the lane is value e of the first
 * two fours and value e of the last two; neighbours: the pairs are within the fours. */
template <int T, bool INTER>
struct RotPiece {
    int q[4];
    bool live, turned;

    __device__ __forceinline__ RotPiece(const RotArgs &a, int lane)
    {
        turned = lane * 8 < a.half;
        live = lane * 16 < a.dim;
        const int n = turned ? a.half / 8 : (a.dim - 2 * a.half) / 16; /* lanes of its region */
        const int at = turned ? lane : lane - a.half / 8, base = turned ? 0 : 2 * a.half;
        constexpr bool F32 = T == PARASON_DTYPE_F32;
        if (!INTER && turned) {
            q[0] = F32 ? 4 * at : 8 * at, q[1] = F32 ? 4 * (at + n) : q[0] + 4;
            q[2] = a.half + q[0], q[3] = a.half + q[1];
        } else if (F32) {
            for (int i = 0; i < 4; ++i) q[i] = base + 4 * (at + i * n);
        } else {
            q[0] = base + 8 * at, q[1] = q[0] + 4, q[2] = base + 8 * (at + n), q[3] = q[2] + 4;
        }
    }
};

template <int T, bool INTER>
__device__ __forceinline__ void rot_load(const char *head, const RotPiece<T, INTER> &p, bool wide, float *x)
{
    const char *const first = head + p.q[0] * type_bytes<T>(), *const last = head + p.q[2] * type_bytes<T>();
    load8<T>(first, 0, p.q[1] - p.q[0], true, wide, x);
    load8<T>(last, 0, p.q[3] - p.q[2], true, wide, x + 8);
}

template <int T, bool INTER>
__device__ __forceinline__ void rot_store(char *head, const RotPiece<T, INTER> &p, bool wide, const float *x)
{
    char *const first = head + p.q[0] * type_bytes<T>(), *const last = head + p.q[2] * type_bytes<T>();
    store8<T>(first, 0, p.q[1] - p.q[0], true, wide, x);
    store8<T>(last, 0, p.q[3] - p.q[2], true, wide, x + 8);
}

/* 16 values of LDS at the lane's places. */
template <class P>
__device__ __forceinline__ void rot_gather(const float *from, const P &p, float *x)
{
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float4 v = *reinterpret_cast<const float4 *>(from + p.q[i]);
        x[4 * i] = v.x, x[4 * i + 1] = v.y, x[4 * i + 2] = v.z, x[4 * i + 3] = v.w;
    }
}

/* DIRECTION 1: by the token's angles, -1: back */
template <int DIRECTION, int T, bool INTER>
__device__ __forceinline__ void rot_turn(float *x, const RotPiece<T, INTER> &p, const float2 *turns)
{
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const float2 cs = turns[INTER ? p.q[e / 2] / 2 + (e & 1) : p.q[e / 4] + (e & 3)];
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
    const RotPiece<T, INTER> p(a, lane);
    const int q_units = n * a.q_heads, units = q_units + n * a.k_heads, step = ROT_THREADS >> a.group_log;
    for (int u = (int)threadIdx.x >> a.group_log; u < units; u += step) {
        const RotUnit v = rot_unit(a, u, q_units);
        const int64_t t = t0 + v.token;
        float x[16] = {};
        if (p.live) {
            rot_load<T>(rot_head<T>(a.x, v, t), p, a.x.wide, x);
        }
        float sum = 0.0f;
#pragma unroll
        for (int e = 0; e < 16; ++e) sum = __builtin_fmaf(x[e], x[e], sum);
        const float r = rsqrtf(__builtin_fmaf(group_sum(sum, a.group_log), a.inv_dim, a.eps));
        if (!p.live) continue;
        float w[16];
        rot_gather(s.w[v.is_k], p, w);
#pragma unroll
        for (int e = 0; e < 16; ++e) x[e] *= r * w[e];
        if (p.turned) rot_turn<1>(x, p, s.turns + v.token * a.half);
        if (a.positions[t] < 0) {
#pragma unroll
            for (int e = 0; e < 16; ++e) x[e] = 0.0f;
        }
        rot_store<T>(rot_head<T>(a.y, v, t), p, a.y.wide, x);
    }
}

/* The same with the gradient turned back; a lane always has the same values of
 * its heads and keeps its sums of the weights' gradients in registers. */
template <int T, bool INTER>
__global__ void __launch_bounds__(ROT_THREADS, 4) qk_norm_rotate_grad(RotArgs a)
{
    __shared__ RotLds s;
    __shared__ __attribute__((aligned(16))) float sums[ROT_THREADS * 16];
    const int lane = (int)threadIdx.x & ((1 << a.group_log) - 1), groups = ROT_THREADS >> a.group_log;
    const int mine = (int)threadIdx.x >> a.group_log;
    const RotPiece<T, INTER> p(a, lane);
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
                rot_load<T>(rot_head<T>(a.x, v, t), p, a.x.wide, x);
                rot_load<T>(rot_head<T>(a.g, v, t), p, a.g.wide, g);
                if (p.turned) rot_turn<-1>(g, p, s.turns + v.token * a.half);
            }
            float sum = 0.0f, dot = 0.0f, gw[16];
            if (p.live) rot_gather(s.w[v.is_k], p, gw);
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                gw[e] = p.live && there ? gw[e] * g[e] : 0.0f; /* (padding: whatever the weight is) */
                sum = __builtin_fmaf(x[e], x[e], sum);
                dot = __builtin_fmaf(gw[e], x[e], dot);
            }
            const float r = rsqrtf(__builtin_fmaf(group_sum(sum, a.group_log), a.inv_dim, a.eps));
            dot = group_sum(dot, a.group_log) * r * a.inv_dim;
            dot = r == 0.0f ? 0.0f : dot; /* (a head without a length has no gradient, also where this sum is infinite) */
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
            rot_store<T>(rot_head<T>(a.y, v, t), p, a.y.wide, x);
        }
    }
    /* the block's groups of lanes, added in their order */
#pragma unroll
    for (int which = 0; which < 2; ++which) {
        __syncthreads();
        if (p.live) {
#pragma unroll
            for (int i = 0; i < 4; ++i)
                *reinterpret_cast<float4 *>(&sums[mine * a.dim + p.q[i]]) =
                    make_float4(acc[which][4 * i], acc[which][4 * i + 1], acc[which][4 * i + 2], acc[which][4 * i + 3]);
        }
        __syncthreads();
        for (int d = (int)threadIdx.x; d < a.dim; d += ROT_THREADS) {
            float x = 0.0f;
#pragma unroll 16
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
