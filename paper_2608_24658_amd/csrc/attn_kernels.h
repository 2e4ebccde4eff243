/*
 * attn_kernels.h -- attention of a tree of tokens over the paged cache for
 * gfx950.
 */
#pragma once
#include "kv_common.h"

namespace pk {

struct TreeArgs {
    KvCache c;
    KvRows r;
    const char *q;
    char *out;
    float *lse;
    int64_t q_stride_token, q_stride_head, out_stride_token, out_stride_head;
    const uint64_t *mask;
    int64_t mask_stride;
    const int32_t *tree_lens;
    int32_t mask_words, n_q_heads;
    float scale;
    bool f16;
    int kind;
};

__device__ __forceinline__ float to_f32(const char *p, bool f16)
{
    const uint32_t h = *reinterpret_cast<const uint16_t *>(p);
    return f16 ? f16_to_f32(h) : bf16_to_f32(h);
}

__device__ __forceinline__ float cached(const char *base, int64_t at, int kind)
{
    if (kind == KV_BF16 || kind == KV_F16) return to_f32(base + at * 2, kind == KV_F16);
    float x[4];
    const uint32_t w = (uint8_t)base[at];
    if (kind == KV_FP8) fp8x4_to_f32(w, x);
    else int8x4_to_f32(w, x);
    return x[0];
}

/* One block per (token, query head): 256 positions at a time, a thread for
 * each; then a thread for each value of the head. */
__global__ void __launch_bounds__(256) tree_attention_simple(TreeArgs a)
{
    __shared__ float qs[PARASON_KV_MAX_DIM], ps[256], red[8];
    __shared__ int64_t at_v[256];
    const int64_t row = blockIdx.x / (uint32_t)a.r.max_length;
    const int32_t j = (int32_t)(blockIdx.x % (uint32_t)a.r.max_length);
    const int head = (int)blockIdx.y, kv_head = head / (a.n_q_heads / a.c.n_heads);
    const int tid = (int)threadIdx.x, D = a.c.head_dim;
    const KvRow w = load_row(a.r, a.c, row, false);
    if (!w.out_ok) {
        if (tid == 0) report(a.r, row, PARASON_KV_BAD_ROW);
        return;
    }
    if (j >= w.length) return;
    const int64_t t = w.start + j;
    const int32_t tree = a.mask ? (a.tree_lens ? a.tree_lens[row] : w.length) : 0;
    const bool ok = w.ok && (!a.mask || (tree >= 0 && tree <= w.kv_len && (tree + 63) / 64 <= a.mask_words));
    if (!ok && tid == 0) report(a.r, row, PARASON_KV_BAD_ROW);
    const int32_t base = w.kv_len - tree;
    const int32_t end = !ok ? 0 : (a.mask ? w.kv_len : min(w.kv_len, w.kv_len - w.length + j + 1));
    bool bad = !ok;
    if (tid < D) qs[tid] = to_f32(a.q + (t * a.q_stride_token + head * a.q_stride_head + tid) * 2, a.f16);
    float m = -INFINITY, l = 0.0f, o = 0.0f;
    for (int32_t p0 = 0; p0 < end; p0 += 256) {
        const int32_t p = p0 + tid;
        bool seen = p < end;
        if (seen && p >= base && a.mask)
            seen = (a.mask[t * a.mask_stride + (p - base) / 64] >> ((p - base) & 63)) & 1;
        float s = -INFINITY, vs = 1.0f;
        int64_t av = 0;
        __syncthreads();
        if (seen) {
            int32_t slot;
            const int32_t page = page_of(a.r, a.c, row, p, &slot);
            if (page < 0) {
                report(a.r, row, PARASON_KV_BAD_PAGE);
                s = __uint_as_float(0x7FC00000u);
            } else {
                av = (int64_t)page * a.c.stride_page + (int64_t)slot * a.c.stride_slot + kv_head * a.c.stride_head;
                s = 0.0f;
                for (int d = 0; d < D; ++d) s += qs[d] * cached(a.c.k, av + d, a.kind);
                if (a.c.k_scale) {
                    const int64_t as = (int64_t)page * a.c.scale_stride_page + (int64_t)slot * a.c.scale_stride_slot +
                                       kv_head * a.c.scale_stride_head;
                    s *= a.c.k_scale[as];
                    vs = a.c.v_scale[as];
                }
                s *= a.scale;
            }
        }
        float top = s;
        for (int k = 32; k > 0; k >>= 1) top = fmaxf(top, __shfl_xor(top, k));
        if ((tid & 63) == 0) red[tid >> 6] = top;
        at_v[tid] = seen ? av : -1;
        __syncthreads();
        const float m_new = fmaxf(fmaxf(fmaxf(m, red[0]), red[1]), fmaxf(red[2], red[3]));
        const float ref = m_new == -INFINITY ? 0.0f : m_new;
        const float e = seen ? __expf(s - ref) : 0.0f;
        ps[tid] = e * vs;
        float sum = e;
        for (int k = 32; k > 0; k >>= 1) sum += __shfl_xor(sum, k);
        if ((tid & 63) == 0) red[4 + (tid >> 6)] = sum;
        __syncthreads();
        const float corr = m == -INFINITY ? 0.0f : __expf(m - ref);
        l = l * corr + red[4] + red[5] + red[6] + red[7];
        o *= corr;
        m = m_new;
        if (tid < D)
            for (int k = 0; k < min(256, end - p0); ++k)
                if (at_v[k] >= 0) o += ps[k] * cached(a.c.v, at_v[k] + tid, a.kind);
    }
    if (bad) o = l = __uint_as_float(0x7FC00000u);
    const float r = l == 0.0f ? 0.0f : o / l;
    if (tid < D) {
        uint16_t *dst = reinterpret_cast<uint16_t *>(a.out) + t * a.out_stride_token + head * a.out_stride_head + tid;
        *dst = (uint16_t)(a.f16 ? f32_to_f16(r) : f32_to_bf16(r));
    }
    if (tid == 0 && a.lse) a.lse[t * a.n_q_heads + head] = l == 0.0f ? -INFINITY : m + logf(l);
}

}  // namespace pk
