/*
 * beam_kernels.h -- beam selection and the reordering of what belongs to a
 * beam for gfx950.
 */
#pragma once
#include "kv_common.h"

namespace pk {

constexpr int BEAM_THREADS = 256;

struct BeamArgs {
    const char *logits;
    int64_t vocab, row_bytes, rows;
    const float *scores;
    const parason_decode_state *states;
    int32_t beams;
    double *norm;      /* [rows] score - ln sum exp of the row, NaN: offers no tokens */
    float *new_scores;
    int32_t *parents, *tokens;
};

template <int T>
__device__ __forceinline__ float logit(const char *row, int64_t i)
{
    if (T == PARASON_DTYPE_F32) return reinterpret_cast<const float *>(row)[i];
    const uint32_t h = reinterpret_cast<const uint16_t *>(row)[i];
    return T == PARASON_DTYPE_BF16 ? bf16_to_f32(h) : f16_to_f32(h);
}

template <int T>
__global__ void __launch_bounds__(BEAM_THREADS) beam_norm(BeamArgs a)
{
    __shared__ float red[8];
    const int64_t row = blockIdx.x;
    const char *x = a.logits + row * a.row_bytes;
    float m = -INFINITY;
    bool bad = false;
    for (int64_t i = threadIdx.x; i < a.vocab; i += BEAM_THREADS) {
        const float v = logit<T>(x, i);
        bad = bad || !(v < INFINITY);
        m = fmaxf(m, v);
    }
    for (int k = 32; k > 0; k >>= 1) m = fmaxf(m, __shfl_xor(m, k));
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = m;
    bad = __syncthreads_or(bad);
    m = fmaxf(fmaxf(red[0], red[1]), fmaxf(red[2], red[3]));
    float s = 0.0f;
    if (!bad && m > -INFINITY)
        for (int64_t i = threadIdx.x; i < a.vocab; i += BEAM_THREADS) s += __expf(logit<T>(x, i) - m);
    for (int k = 32; k > 0; k >>= 1) s += __shfl_xor(s, k);
    if ((threadIdx.x & 63) == 0) red[4 + (threadIdx.x >> 6)] = s;
    __syncthreads();
    if (threadIdx.x == 0) {
        const float score = a.scores[row];
        const bool live = isfinite(score) && !bad && m > -INFINITY && !(a.states && a.states[row].flags);
        const double total = (double)red[4] + red[5] + red[6] + red[7];
        a.norm[row] = live ? (double)score - ((double)m + log(total)) : (double)NAN;
    }
}

/* One block per group; a round per beam finds the best candidate behind the
 * one before. */
template <int T>
__global__ void __launch_bounds__(BEAM_THREADS) beam_rounds(BeamArgs a)
{
    __shared__ double best_s[BEAM_THREADS];
    __shared__ int64_t best_i[BEAM_THREADS];
    __shared__ float sc[PARASON_BEAM_MAX];
    const int64_t row0 = (int64_t)blockIdx.x * a.beams;
    if ((int)threadIdx.x < a.beams) sc[threadIdx.x] = a.scores[row0 + threadIdx.x];
    double last_s = (double)INFINITY;
    int64_t last_i = -1;
    for (int k = 0; k < a.beams; ++k) {
        double bs = -(double)INFINITY;
        int64_t bi = -1;
        __syncthreads();
        for (int b = 0; b < a.beams; ++b) {
            const char *x = a.logits + (row0 + b) * a.row_bytes;
            const double norm = a.norm[row0 + b];
            const uint32_t flags = a.states ? a.states[row0 + b].flags : 0u;
            const bool stay = !(flags & PARASON_DECODE_ERROR) && (flags & PARASON_DECODE_DONE) && isfinite(sc[b]);
            if (norm != norm && !stay) continue;
            for (int64_t i = threadIdx.x; i < (stay ? 1 : a.vocab); i += BEAM_THREADS) {
                const double s = stay ? (double)sc[b] : norm + (double)logit<T>(x, i);
                const int64_t id = b * (a.vocab + 1) + (stay ? 0 : i + 1);
                if (!(s > -(double)INFINITY)) continue;
                if ((s < last_s || (s == last_s && id > last_i)) && (s > bs || (s == bs && id < bi))) bs = s, bi = id;
            }
        }
        best_s[threadIdx.x] = bs, best_i[threadIdx.x] = bi;
        __syncthreads();
        for (int o = BEAM_THREADS / 2; o > 0; o >>= 1) {
            if ((int)threadIdx.x < o) {
                const double s = best_s[threadIdx.x + o];
                const int64_t i = best_i[threadIdx.x + o];
                if (i >= 0 && (best_i[threadIdx.x] < 0 || s > best_s[threadIdx.x] ||
                               (s == best_s[threadIdx.x] && i < best_i[threadIdx.x])))
                    best_s[threadIdx.x] = s, best_i[threadIdx.x] = i;
            }
            __syncthreads();
        }
        last_s = best_s[0], last_i = best_i[0];
        if (threadIdx.x == 0) {
            const int64_t r = row0 + k;
            a.new_scores[r] = last_i < 0 ? -INFINITY : (float)last_s;
            a.parents[r] = (int32_t)(last_i < 0 ? r : row0 + last_i / (a.vocab + 1));
            a.tokens[r] = last_i < 0 ? -1 : (int32_t)(last_i % (a.vocab + 1)) - 1;
        }
        if (last_i < 0) last_s = -(double)INFINITY, last_i = INT64_MAX;
    }
}

struct ReorderArgs {
    const int32_t *parents;
    int64_t n_rows;
    int32_t n_arrays;
    parason_beam_array arrays[PARASON_BEAM_ARRAYS];
};

__global__ void __launch_bounds__(256) beam_reorder(ReorderArgs a)
{
    const int64_t row = blockIdx.x;
    const int64_t parent = a.parents[row];
    if (parent < 0 || parent >= a.n_rows) return;
    for (int k = 0; k < a.n_arrays; ++k) {
        const parason_beam_array &x = a.arrays[k];
        const char *src = (const char *)x.src + parent * x.src_stride;
        char *dst = (char *)x.dst + row * x.dst_stride;
        for (int64_t i = threadIdx.x; i < x.row_bytes; i += 256) dst[i] = src[i];
    }
}

}  // namespace pk
