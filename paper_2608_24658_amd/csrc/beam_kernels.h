/*
 * beam_kernels.h -- beam selection and the reordering of what belongs to a
 * beam for gfx950.
 *
 * The selection is one pass over the logits.  A candidate's score, float32(score
 * + float32(logit - lse)), does not fall as its logit rises, so a block takes a
 * chunk of a row into registers, and from these the chunk's maximum, its sum of
 * exponentials and its `beams` largest logits; a block per group then has each
 * row's sum and chooses among the chunks' candidates by their scores.  Rounding
 * can make the scores of different logits equal, and of equal ones the lowest
 * token counts: a chunk also says how large a logit it has left out, and where
 * the score of that one is still among the best, the tokens of the last score
 * are taken from the logits again, in their order.  Bound by the
 * read: 2,048 rows of 50,257 float16 logits and their reordering, 409 MB in
 * all, take 117 us, the scan 70 of them; 256 rows of 151,936 float32 logits 46
 * us.  The beams of one prompt are three launches, 17 us, and the host's checks,
 * 27 in all.
 *
 * The largest of many, by a bound from below: of the threads' own maxima each
 * wave finds the k-th largest, k a quarter of the beams, by counting lanes bit
 * by bit; the least of these over the four waves has at least `beams` values at or above
 * it, and rarely many more.  Those go to a list in LDS, where each counts the
 * ones before it.  A list that overflows (thousands of equal values) is done
 * without: the best, then the best behind it, and so on.
 */
#pragma once
#include <float.h>

#include "kv_common.h"

namespace pk {

constexpr int BEAM_THREADS = 256;
constexpr int BEAM_PER_THREAD = 32;                              /* logits */
constexpr int BEAM_CHUNK = BEAM_THREADS * BEAM_PER_THREAD;
constexpr int BEAM_LIST = 1024;                                  /* candidates of a block */
constexpr int BEAM_ROW_LANES = 8;                                /* that add up the sums of a row's chunks */

struct __attribute__((packed, aligned(2))) Unaligned16 {
    uint32_t w[4];
};

struct BeamCandidate {
    float logit;   /* -inf: none */
    int32_t token;
};

struct BeamChunk {
    float top;     /* the largest logit */
    float below;   /* the largest logit that is less than that of the last candidate, or a little more; -inf: none */
    double sum;    /* of exp(logit - top) */
};

struct BeamArgs {
    const char *logits;
    int64_t vocab, row_bytes;
    int32_t dtype;
    const float *scores;
    const parason_decode_state *states;
    int32_t beams, chunks;
    FastDiv chunks_div;
    int32_t chunk_pieces;     /* 16-byte pieces of a chunk: the row's, evenly */
    int64_t chunk_tokens;     /* logits of these */
    BeamChunk *sums;          /* [rows][chunks] */
    BeamCandidate *best;      /* [rows][chunks][beams], best first */
    float *new_scores;
    int32_t *parents, *tokens;
};

/* What a row offers. */
enum : int { BEAM_NONE = 0, BEAM_TOKENS, BEAM_STAYS };

__device__ __forceinline__ int beam_offers(const BeamArgs &a, int64_t row, float score)
{
    if (!(score > -INFINITY && score < INFINITY)) return BEAM_NONE;
    if (!a.states) return BEAM_TOKENS;
    const uint32_t f = a.states[row].flags;
    return (f & PARASON_DECODE_ERROR) ? BEAM_NONE : (f & PARASON_DECODE_DONE) ? BEAM_STAYS : BEAM_TOKENS;
}

/* Floats as integers of the same order. */
__device__ __forceinline__ uint32_t in_order(float x)
{
    const uint32_t u = __float_as_uint(x);
    return u & 0x80000000u ? ~u : u | 0x80000000u;
}

__device__ __forceinline__ float from_order(uint32_t k) { return __uint_as_float(k & 0x80000000u ? k & 0x7FFFFFFFu : ~k); }

/* A value that at least k of the wave's lanes (k <= 64) are not below, to 16
 * bits, and above -inf. */
__device__ __forceinline__ float wave_kth(float x, int k)
{
    const uint32_t key = in_order(x);
    uint32_t t = 0u;
#pragma unroll
    for (int b = 31; b >= 16; --b) {
        const uint32_t trial = t | (1u << b);
        if (__popcll(__ballot(key >= trial)) >= k) t = trial;
    }
    const uint32_t least = 0x00800000u; /* -FLT_MAX */
    return from_order(t < least ? least : t);
}

/* A value that at least n of the block's threads' values are not below (or
 * -FLT_MAX).  red: 8 floats. */
__device__ __forceinline__ float block_bound(float x, int n, float *red)
{
    const int wave = (int)threadIdx.x >> 6;
    const float t = wave_kth(x, (n + 3) / 4);
    if ((threadIdx.x & 63) == 0) red[wave] = t;
    __syncthreads();
    const float least = fminf(fminf(red[0], red[1]), fminf(red[2], red[3]));
    if (least > -FLT_MAX) return least;
    /* a wave with too few values: one that has n by itself may do */
    const float u = wave_kth(x, n);
    if ((threadIdx.x & 63) == 0) red[4 + wave] = u;
    __syncthreads();
    return fmaxf(fmaxf(red[4], red[5]), fmaxf(red[6], red[7]));
}

/* A larger key is the better candidate: the larger logit, of equal ones (zeros of either sign are equal) the lower token. */
__device__ __forceinline__ uint64_t beam_key(float logit, int32_t token)
{
    return ((uint64_t)in_order(logit + 0.0f) << 32) | (uint32_t)~token;
}

/* The sum of exponentials is that of the products logit * log2(e), of which the second part makes up for the rounding
 * of the first: alike in every term, it would not average out. */
constexpr float LOG2E_HI = 1.44269502f, LOG2E_LO = 1.92596299e-8f;

/* The largest logit of the type below x, or a little more (of float16's smallest). */
template <int T>
__device__ __forceinline__ float logit_below(float x)
{
    /* in_order() of 16-bit logits: bits that are all zero, or of negative ones all one */
    constexpr uint32_t rest = T == PARASON_DTYPE_F32 ? 0u : T == PARASON_DTYPE_BF16 ? 0xFFFFu : 0x1FFFu;
    const uint32_t k = in_order(x) - 1u;
    return from_order((k & 0x80000000u) ? k & ~rest : (k & rest) == rest ? k : (k & ~rest) - 1u);
}

__device__ __forceinline__ int lanes_below(uint64_t mask)
{
    return (int)__builtin_amdgcn_mbcnt_hi((uint32_t)(mask >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)mask, 0u));
}

/* Six waves a SIMD: with the registers of five 77 us against 68 for 2,048 rows of 50,257 float16 logits, traced in turn. */
template <int T>
__global__ void __launch_bounds__(BEAM_THREADS, 6) beam_scan(BeamArgs a)
{
    constexpr int ES = T == PARASON_DTYPE_F32 ? 4 : 2, VE = 16 / ES, NV = BEAM_PER_THREAD / VE;
    __shared__ float red[12];
    __shared__ double red_sum[4];
    __shared__ uint32_t last_order, below_order;
    __shared__ __attribute__((aligned(16))) uint64_t list[BEAM_LIST + 2]; /* order of the logit, and of the token from the last */
    __shared__ int32_t n_list;
    const uint32_t chunk = blockIdx.x % (uint32_t)a.chunks;
    const int64_t row = blockIdx.x / (uint32_t)a.chunks;
    const int tid = (int)threadIdx.x;
    BeamCandidate *const best = a.best + (int64_t)blockIdx.x * a.beams; /* (blocks are counted as [rows][chunks]) */
    const char *const x = a.logits + row * a.row_bytes;
    if (beam_offers(a, row, a.scores[row]) != BEAM_TOKENS) return;
    /* 16 bytes at a time from the row's first logit on, at whatever alignment that has: which logits a lane adds up, and
     * so a row's sum, does not depend on where the row lies */
    const int64_t e0 = ((int64_t)chunk * a.chunk_pieces + tid) * VE;
    const int64_t next = (int64_t)(chunk + 1) * a.chunk_pieces * VE, end = next < a.vocab ? next : a.vocab;
    uint4 raw[NV];
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int64_t e = e0 + (int64_t)i * BEAM_THREADS * VE;
        if (e + VE <= end) {
            const Unaligned16 p = *reinterpret_cast<const Unaligned16 *>(x + e * ES);
            raw[i] = make_uint4(p.w[0], p.w[1], p.w[2], p.w[3]);
        } else {
            uint32_t w[4];
            for (int j = 0; j < 4; ++j) {
                if (ES == 4) {
                    w[j] = e + j < end ? reinterpret_cast<const uint32_t *>(x)[e + j] : 0xFF800000u;
                } else {
                    const uint32_t none = T == PARASON_DTYPE_BF16 ? 0xFF80u : 0xFC00u;
                    const int64_t p = e + 2 * j;
                    const uint32_t lo = p < end ? reinterpret_cast<const uint16_t *>(x)[p] : none;
                    const uint32_t hi = p + 1 < end ? reinterpret_cast<const uint16_t *>(x)[p + 1] : none;
                    w[j] = lo | (hi << 16);
                }
            }
            raw[i] = make_uint4(w[0], w[1], w[2], w[3]);
        }
    }
    float v[BEAM_PER_THREAD];
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const uint32_t w[4] = {raw[i].x, raw[i].y, raw[i].z, raw[i].w};
#pragma unroll
        for (int j = 0; j < VE; ++j)
            v[i * VE + j] = ES == 4 ? __uint_as_float(w[j & 3])
                            : T == PARASON_DTYPE_BF16 ? bf16_to_f32((w[(j / 2) & 3] >> (16 * (j & 1))) & 0xFFFFu)
                                                      : f16_to_f32((w[(j / 2) & 3] >> (16 * (j & 1))) & 0xFFFFu);
    }
    auto token_of = [&](int i) { return (int32_t)(e0 + (int64_t)(i / VE) * BEAM_THREADS * VE + i % VE); };
    float mine = v[0];
#pragma unroll
    for (int i = 1; i < BEAM_PER_THREAD; ++i) mine = fmaxf(mine, v[i]);
    if (!(mine == mine)) mine = -INFINITY; /* nothing but NaN: the sum tells */
    float m = mine;
#pragma unroll
    for (int k = 32; k > 0; k >>= 1) m = fmaxf(m, __shfl_xor(m, k));
    if ((tid & 63) == 0) red[8 + (tid >> 6)] = m;
    if (tid == 0) n_list = 0, below_order = 0u;
    const float bound = block_bound(mine, a.beams, red);
    m = fmaxf(fmaxf(red[8], red[9]), fmaxf(red[10], red[11]));
    /* ---- sum */
    const float ref = m == -INFINITY ? 0.0f : m;
    float mine_sum = 0.0f;
#pragma unroll
    for (int i = 0; i < BEAM_PER_THREAD; ++i) {
        const float d = v[i] - ref;
        mine_sum += __builtin_amdgcn_exp2f(__builtin_fmaf(d, LOG2E_HI, d * LOG2E_LO));
    }
#pragma unroll
    for (int k = 32; k > 0; k >>= 1) mine_sum += __shfl_xor(mine_sum, k);
    /* (double beyond a wave: the logarithm is rounded to float32, and the order of adding should not show in it) */
    if ((tid & 63) == 0) red_sum[tid >> 6] = (double)mine_sum;
    /* ---- candidates */
    int count = 0;
#pragma unroll
    for (int i = 0; i < BEAM_PER_THREAD; ++i) count += __popcll(__ballot(v[i] >= bound));
    if (count > 0) { /* the same for the whole wave */
        int base = 0;
        if ((tid & 63) == 0) base = atomicAdd(&n_list, count);
        base = __builtin_amdgcn_readfirstlane(base);
#pragma unroll
        for (int i = 0; i < BEAM_PER_THREAD; ++i) {
            const uint64_t b = __ballot(v[i] >= bound);
            if (b == 0) continue;
            const int at = base + lanes_below(b);
            if (v[i] >= bound && at < BEAM_LIST) list[at] = beam_key(v[i], token_of(i));
            base += __popcll(b);
        }
    }
    __syncthreads();
    const int n = n_list;
    auto record = [&](float below) {
        a.sums[blockIdx.x] = BeamChunk{fmaxf(fmaxf(red[8], red[9]), fmaxf(red[10], red[11])), below,
                                       red_sum[0] + red_sum[1] + red_sum[2] + red_sum[3]};
    };
    if (n <= BEAM_LIST) {
        if (tid < 2) list[n + tid] = 0;      /* (before everything) */
        __syncthreads();
        uint64_t next = 0;                   /* the best that is no candidate, at the thread that ranks it */
        for (int c = tid; c < n; c += BEAM_THREADS) {
            const uint64_t me = list[c];
            int before = 0;
            for (int k = 0; k < n; k += 2) {
                const ulonglong2 o = *reinterpret_cast<const ulonglong2 *>(&list[k]);
                before += (o.x > me) + (o.y > me);
            }
            if (before < a.beams) best[before] = BeamCandidate{from_order((uint32_t)(me >> 32)), (int32_t)~(uint32_t)me};
            if (before == a.beams - 1) last_order = (uint32_t)(me >> 32);
            if (before == a.beams) next = me;
        }
        if (tid >= n && tid < a.beams) best[tid] = BeamCandidate{-INFINITY, -1};
        /* what is left out: of the list, or else below the bound, where there is anything below it */
        const float rest = bound > -FLT_MAX ? logit_below<T>(bound) : -INFINITY;
        if (n <= a.beams) {
            if (tid == 0) record(rest);
            return;
        }
        __syncthreads();
        if (__ballot(next != 0) == 0) return;
        /* the wave that has it; where it equals the last candidate, what comes behind those that do */
        const uint32_t last = last_order;
        uint32_t below = (uint32_t)(next >> 32);
        if (__ballot(next != 0 && below == last)) {
            for (int c = tid & 63; c < n; c += 64) {
                const uint32_t o = (uint32_t)(list[c] >> 32);
                if (o < last) atomicMax(&below_order, o);
            }
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            __builtin_amdgcn_wave_barrier();
            below = below_order;
        }
        if (next != 0) record(below != 0u ? from_order(below) : rest);
        return;
    }
    /* too many equal ones: one after the other */
    BeamCandidate last{INFINITY, -1};
    for (int k = 0; k < a.beams; ++k) {
        BeamCandidate b{-INFINITY, INT32_MAX};
#pragma unroll
        for (int i = 0; i < BEAM_PER_THREAD; ++i) {
            const int32_t t = token_of(i);
            if ((v[i] < last.logit || (v[i] == last.logit && t > last.token)) && v[i] > b.logit) b = BeamCandidate{v[i], t};
        }
        /* a thread's own equal ones come in the order of their tokens */
#pragma unroll
        for (int o = 32; o > 0; o >>= 1) {
            const float f = __shfl_xor(b.logit, o);
            const int32_t t = __shfl_xor(b.token, o);
            if (f > b.logit || (f == b.logit && t < b.token)) b = BeamCandidate{f, t};
        }
        __syncthreads();
        BeamCandidate *const heads = reinterpret_cast<BeamCandidate *>(list);
        if ((tid & 63) == 0) heads[tid >> 6] = b;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            const BeamCandidate o = heads[w];
            if (o.logit > b.logit || (o.logit == b.logit && o.token < b.token)) b = o;
        }
        if (tid == 0) best[k] = BeamCandidate{b.logit, b.logit == -INFINITY ? -1 : b.token};
        last = b;
    }
    float below = -INFINITY;
#pragma unroll
    for (int i = 0; i < BEAM_PER_THREAD; ++i)
        if (v[i] < last.logit) below = fmaxf(below, v[i]);
#pragma unroll
    for (int k = 32; k > 0; k >>= 1) below = fmaxf(below, __shfl_xor(below, k));
    __syncthreads();
    if ((tid & 63) == 0) red[tid >> 6] = below;
    __syncthreads();
    if (tid == 0) record(fmaxf(fmaxf(red[0], red[1]), fmaxf(red[2], red[3])));
}

struct BeamScored {
    float score;
    int64_t place; /* (beam of the group, token + 1) */
};

__device__ __forceinline__ bool beam_before(const BeamScored &a, const BeamScored &b)
{
    return a.score > b.score || (a.score == b.score && a.place < b.place);
}

__device__ __forceinline__ float beam_logit(const BeamArgs &a, int64_t row, int64_t token)
{
    const char *x = a.logits + row * a.row_bytes;
    if (a.dtype == PARASON_DTYPE_F32) return reinterpret_cast<const float *>(x)[token];
    const uint32_t h = reinterpret_cast<const uint16_t *>(x)[token];
    return a.dtype == PARASON_DTYPE_BF16 ? bf16_to_f32(h) : f16_to_f32(h);
}

/* One block per group.  The chunks' candidates are lists, best first: a bound
 * comes from the heads of the lists, and each list is then read as far as it
 * reaches.  Bound by latency: a chain of four memory rounds and two rankings
 * in LDS, so that one block does a group of 32 beams of 7 chunks as quickly as
 * several would. */
__global__ void __launch_bounds__(BEAM_THREADS) beam_choose(BeamArgs a)
{
    __shared__ float red[8];
    __shared__ float score[PARASON_BEAM_MAX];
    __shared__ float lse[PARASON_BEAM_MAX];
    __shared__ float left_out[PARASON_BEAM_MAX]; /* no candidate that a list of the row lacks has a larger score but for equal logits */
    __shared__ int32_t offers[PARASON_BEAM_MAX];
    __shared__ BeamScored list[BEAM_LIST];
    __shared__ BeamScored chosen[PARASON_BEAM_MAX];
    __shared__ int32_t n_list, n_live, found[4];
    const int tid = (int)threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int64_t row0 = (int64_t)blockIdx.x * a.beams;
    const BeamScored none{-INFINITY, INT64_MAX};
    if (tid == 0) n_list = n_live = 0;
    if (tid < PARASON_BEAM_MAX) chosen[tid] = none;
    __syncthreads();
    /* a token's score: three float32 roundings, the same wherever it is worked out */
    auto scored = [&](int b, float logit) { return score[b] + (logit - lse[b]); };
    for (int b0 = 0; b0 < a.beams; b0 += BEAM_THREADS / BEAM_ROW_LANES) {
        const int b = b0 + tid / BEAM_ROW_LANES, part = tid % BEAM_ROW_LANES;
        const bool there = b < a.beams;
        const int64_t row = row0 + (there ? b : 0);
        const float sc = a.scores[row];
        const int what = there ? beam_offers(a, row, sc) : BEAM_NONE;
        float m = -INFINITY, below = -INFINITY;
        double s = 0.0; /* an empty chunk has the maximum -inf and the sum 0 */
        if (what == BEAM_TOKENS) {
            for (int c = part; c < a.chunks; c += BEAM_ROW_LANES) {
                m = fmaxf(m, a.sums[row * a.chunks + c].top);
                below = fmaxf(below, a.sums[row * a.chunks + c].below);
            }
        }
#pragma unroll
        for (int k = BEAM_ROW_LANES / 2; k > 0; k >>= 1) {
            m = fmaxf(m, __shfl_xor(m, k));
            below = fmaxf(below, __shfl_xor(below, k));
        }
        if (what == BEAM_TOKENS && m > -INFINITY) {
            for (int c = part; c < a.chunks; c += BEAM_ROW_LANES) {
                const BeamChunk q = a.sums[row * a.chunks + c];
                s += q.sum * exp((double)q.top - (double)m);
            }
        }
#pragma unroll
        for (int k = BEAM_ROW_LANES / 2; k > 0; k >>= 1) s += __shfl_xor(s, k);
        if (there && part == 0) {
            /* NaN or +inf among the logits: s is NaN; nothing but -inf: no sum */
            const bool tokens = what == BEAM_TOKENS && m > -INFINITY && s < (double)INFINITY;
            score[b] = sc, offers[b] = tokens || what == BEAM_STAYS ? what : BEAM_NONE;
            lse[b] = tokens ? m + logf((float)s) : 0.0f;
            left_out[b] = tokens ? scored(b, below) : -INFINITY;
            if (tokens) atomicAdd(&n_live, 1);
        }
    }
    __syncthreads();
    const uint32_t lists = (uint32_t)a.chunks * (uint32_t)a.beams;
    const BeamCandidate *const best = a.best + row0 * lists;
    /* The score of entry k of list i, read as q (-inf: no candidate); a finished row has one, in its first list. */
    auto score_of = [&](uint32_t i, uint32_t k, const BeamCandidate &q) {
        const uint32_t b = div_by(i, a.chunks_div);
        const bool first = k == 0 && i == b * (uint32_t)a.chunks;
        return offers[b] == BEAM_TOKENS ? scored((int)b, q.logit) : offers[b] == BEAM_STAYS && first ? score[b] : -INFINITY;
    };
    auto place_of = [&](uint32_t i, const BeamCandidate &q) {
        const uint32_t b = div_by(i, a.chunks_div);
        return (int64_t)b * (a.vocab + 1) + (offers[b] == BEAM_TOKENS ? q.token + 1 : 0);
    };
    /* The bound, from the first entries of every list, some 64 for each beam (a power of two of every list).
     * Neighbouring entries, which are much alike, go to different threads and waves: it is the least of the waves'. */
    const uint32_t live = (uint32_t)n_live * (uint32_t)a.chunks;
    uint32_t depth_log = 0;
    while (live > 0 && (2u << depth_log) <= (uint32_t)a.beams && (live << (depth_log + 1)) <= 64u * (uint32_t)a.beams) ++depth_log;
    const uint32_t entries = lists << depth_log, depth_mask = (1u << depth_log) - 1u;
    float mine = -INFINITY;
    for (uint32_t i0 = lane * 4 + wave; i0 < entries; i0 += 2 * BEAM_THREADS) {
        const uint32_t i1 = i0 + BEAM_THREADS < entries ? i0 + BEAM_THREADS : i0;
        const BeamCandidate q0 = best[(int64_t)(i0 >> depth_log) * a.beams + (i0 & depth_mask)];
        const BeamCandidate q1 = best[(int64_t)(i1 >> depth_log) * a.beams + (i1 & depth_mask)];
        mine = fmaxf(mine, score_of(i0 >> depth_log, i0 & depth_mask, q0));
        mine = fmaxf(mine, score_of(i1 >> depth_log, i1 & depth_mask, q1));
    }
    const float bound = block_bound(mine, a.beams, red);
    /* ---- what reaches it */
    for (uint32_t i = tid; i < lists; i += BEAM_THREADS) {
        bool more = true;
        for (int k0 = 0; more && k0 < a.beams; k0 += 4) {
            BeamCandidate q[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) q[j] = best[(int64_t)i * a.beams + (k0 + j < a.beams ? k0 + j : k0)];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                if (!more) continue;
                const float sc = score_of(i, (uint32_t)(k0 + j), q[j]);
                more = k0 + j < a.beams && sc >= bound;
                if (!more) continue;
                const int at = atomicAdd(&n_list, 1);
                if (at < BEAM_LIST) list[at] = BeamScored{sc, place_of(i, q[j])};
            }
        }
    }
    __syncthreads();
    const int n = n_list;
    if (n <= BEAM_LIST) {
        for (int i = tid; i < n; i += BEAM_THREADS) {
            const BeamScored me = list[i];
            int before = 0;
            for (int k = 0; k < n; ++k) before += beam_before(list[k], me);
            if (before < a.beams) chosen[before] = me;
        }
    } else {
        /* too many equal ones: one after the other */
        BeamScored last{INFINITY, -1};
        for (int k = 0; k < a.beams; ++k) {
            BeamScored b = none;
            for (uint32_t i = tid; i < lists; i += BEAM_THREADS)
                for (int j = 0; j < a.beams; ++j) {
                    const BeamCandidate q = best[(int64_t)i * a.beams + j];
                    const BeamScored c{score_of(i, (uint32_t)j, q), place_of(i, q)};
                    if (c.score > -INFINITY && beam_before(last, c) && beam_before(c, b)) b = c;
                }
#pragma unroll
            for (int o = 32; o > 0; o >>= 1) {
                const BeamScored q{__shfl_xor(b.score, o), (int64_t)__shfl_xor((long long)b.place, o)};
                if (beam_before(q, b)) b = q;
            }
            __syncthreads();
            if (lane == 0) list[wave] = b;
            __syncthreads();
#pragma unroll
            for (int w = 0; w < 4; ++w)
                if (beam_before(list[w], b)) b = list[w];
            if (tid == 0) chosen[k] = b;
            last = b;
        }
    }
    __syncthreads();
    /* ---- the last score again, where a list may lack a lower token of it (the ones above it are all there: a list that
     * lacks a candidate has `beams` that are no worse) */
    const float cut = chosen[a.beams - 1].score;
    if (__ballot(lane < a.beams && cut > -INFINITY && left_out[lane] >= cut)) { /* the same in every wave */
        int have = __popcll(__ballot(lane < a.beams && chosen[lane].score > cut));
        __syncthreads();
        for (int b = 0; b < a.beams && have < a.beams; ++b) {
            const int64_t row = row0 + b;
            if (offers[b] == BEAM_STAYS && score[b] == cut) {
                if (tid == 0) chosen[have] = BeamScored{cut, (int64_t)b * (a.vocab + 1)};
                ++have;
            }
            if (offers[b] != BEAM_TOKENS) continue;
            for (int c = 0; c < a.chunks && have < a.beams; ++c) {
                if (scored(b, a.sums[row * a.chunks + c].top) < cut) continue;
                const int64_t t0 = (int64_t)c * a.chunk_tokens;
                const int64_t t1 = t0 + a.chunk_tokens < a.vocab ? t0 + a.chunk_tokens : a.vocab;
                for (int64_t t = t0; t < t1 && have < a.beams; t += BEAM_THREADS) {
                    const bool hit = t + tid < t1 && scored(b, beam_logit(a, row, t + tid)) == cut;
                    const uint64_t hits = __ballot(hit);
                    __syncthreads(); /* (the last round's counts have been read) */
                    if (lane == 0) found[wave] = __popcll(hits);
                    __syncthreads();
                    int at = have + lanes_below(hits);
                    for (int w = 0; w < wave; ++w) at += found[w];
                    if (hit && at < a.beams) chosen[at] = BeamScored{cut, (int64_t)b * (a.vocab + 1) + t + tid + 1};
                    have += found[0] + found[1] + found[2] + found[3];
                }
            }
        }
        __syncthreads();
    }
    if (tid >= a.beams) return;
    const BeamScored r = chosen[tid];
    const bool empty = r.place == INT64_MAX;
    const int64_t b = empty ? tid : r.place / (a.vocab + 1);
    a.new_scores[row0 + tid] = r.score;
    a.parents[row0 + tid] = (int32_t)(row0 + b);
    a.tokens[row0 + tid] = empty ? -1 : (int32_t)(r.place - b * (a.vocab + 1)) - 1;
}

/* ---- reordering ---- */

constexpr int REORDER_THREADS = 256;
constexpr int64_t REORDER_SEGMENT = 16384; /* bytes of a row that a block copies: four 16-byte pieces a thread */
constexpr int64_t REORDER_SMALL = 1024;    /* rows of up to this many bytes share a block */

struct ReorderArgs {
    const int32_t *parents;
    int64_t n_rows;
    int32_t n_arrays, n_small, blocks_per_row;
    parason_beam_array arrays[PARASON_BEAM_ARRAYS]; /* the small ones first */
    int32_t first_block[PARASON_BEAM_ARRAYS];       /* of a row, for the others */
    uint8_t width[PARASON_BEAM_ARRAYS];             /* bytes of a piece: what every row's two ends are aligned to */
};

template <typename U, int NT>
__device__ __forceinline__ void copy_pieces(char *dst, const char *src, int64_t lo, int64_t hi, int t)
{
    /* lo and hi in bytes, lo a multiple of the piece; a rest shorter than a piece goes byte by byte */
    constexpr int64_t S = sizeof(U);
    const int64_t n = (hi - lo) / S;
    const U *s = reinterpret_cast<const U *>(src + lo);
    U *d = reinterpret_cast<U *>(dst + lo);
    int64_t i = t;
    for (; i + 3 * NT < n; i += 4 * NT) {
        const U a = s[i], b = s[i + NT], c = s[i + 2 * NT], e = s[i + 3 * NT];
        d[i] = a, d[i + NT] = b, d[i + 2 * NT] = c, d[i + 3 * NT] = e;
    }
    for (; i < n; i += NT) d[i] = s[i];
    for (int64_t k = lo + n * S + t; k < hi; k += NT) dst[k] = src[k];
}

template <int NT>
__device__ __forceinline__ void copy_row(char *dst, const char *src, int64_t lo, int64_t hi, int width, int t)
{
    if (width == 16) copy_pieces<uint4, NT>(dst, src, lo, hi, t);
    else if (width == 4) copy_pieces<uint32_t, NT>(dst, src, lo, hi, t);
    else copy_pieces<uint8_t, NT>(dst, src, lo, hi, t);
}

/* A copy, bound by memory; one launch for all arrays, whose small ones (states,
 * mask rows) share a block so that they do not each need one. */
__global__ void __launch_bounds__(REORDER_THREADS) beam_reorder(ReorderArgs a)
{
    const int64_t row = blockIdx.x / (uint32_t)a.blocks_per_row;
    const int32_t part = (int32_t)(blockIdx.x % (uint32_t)a.blocks_per_row);
    const int64_t parent = a.parents[row];
    if (parent < 0 || parent >= a.n_rows) return;
    if (part == 0 && a.n_small > 0) { /* a wave an array */
        for (int k = (int)threadIdx.x >> 6; k < a.n_small; k += REORDER_THREADS / 64) {
            const parason_beam_array &x = a.arrays[k];
            copy_row<64>((char *)x.dst + row * x.dst_stride, (const char *)x.src + parent * x.src_stride, 0, x.row_bytes,
                         a.width[k], (int)threadIdx.x & 63);
        }
        return;
    }
    int k = a.n_small;
    while (k + 1 < a.n_arrays && part >= a.first_block[k + 1]) ++k;
    const parason_beam_array &x = a.arrays[k];
    const int64_t lo = (part - a.first_block[k]) * REORDER_SEGMENT;
    const int64_t hi = lo + REORDER_SEGMENT < x.row_bytes ? lo + REORDER_SEGMENT : x.row_bytes;
    copy_row<REORDER_THREADS>((char *)x.dst + row * x.dst_stride, (const char *)x.src + parent * x.src_stride, lo, hi,
                              a.width[k], (int)threadIdx.x);
}

}  // namespace pk
