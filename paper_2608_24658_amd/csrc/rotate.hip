/*
 * rotate.hip -- C-ABI of the norm and rotation of queries and keys (kernels in
 * rotate_kernels.h).
 */
#include "kv_abi.h"
#include "rotate_kernels.h"

using abi::aligned;

namespace {

typedef void (*RotKernel)(pk::RotArgs);

template <int T>
RotKernel pick(bool inter, bool grad)
{
    return grad ? (inter ? pk::qk_norm_rotate_grad<T, true> : pk::qk_norm_rotate_grad<T, false>)
                : (inter ? pk::qk_norm_rotate<T, true> : pk::qk_norm_rotate<T, false>);
}

int check_sizes(const parason_rotate *r)
{
    if (!r) return PARASON_ERR_NULL;
    if (r->n_tokens < 0 || r->n_tokens > INT32_MAX || r->n_q_heads < 0 || r->n_q_heads > PARASON_KV_MAX_HEADS ||
        r->n_k_heads < 0 || r->n_k_heads > PARASON_KV_MAX_HEADS || r->head_dim < 16 || r->head_dim > PARASON_KV_MAX_DIM ||
        r->head_dim % 16 != 0 || r->n_turned < 0 || r->n_turned > r->head_dim || r->n_turned % 16 != 0)
        return PARASON_ERR_SIZE;
    return PARASON_OK;
}

int64_t elem_of(int32_t dtype) { return dtype == PARASON_DTYPE_F32 ? 4 : 2; }

/* The heads of a call's tokens; `work`: there is something to read. */
int check_heads(const parason_rotate *r, const parason_heads *h, pk::RotHeads *o)
{
    if (!h) return PARASON_ERR_NULL;
    if (!abi::stride_fits(h->q_stride_token, r->n_tokens) || !abi::stride_fits(h->q_stride_head, r->n_q_heads) ||
        !abi::stride_fits(h->k_stride_token, r->n_tokens) || !abi::stride_fits(h->k_stride_head, r->n_k_heads))
        return PARASON_ERR_SIZE;
    if (r->n_tokens > 0 && ((r->n_q_heads > 0 && !h->q) || (r->n_k_heads > 0 && !h->k))) return PARASON_ERR_NULL;
    const int64_t e = elem_of(r->dtype);
    if (!aligned(h->q, e) || !aligned(h->k, e)) return PARASON_ERR_ALIGN;
    o->q = (char *)h->q, o->k = (char *)h->k;
    o->q_token = h->q_stride_token, o->q_head = h->q_stride_head, o->k_token = h->k_stride_token, o->k_head = h->k_stride_head;
    auto wide = [&](const void *p, int32_t heads, int64_t token, int64_t head) {
        return heads == 0 || (aligned(p, 16) && token * e % 16 == 0 && head * e % 16 == 0);
    };
    o->wide = wide(h->q, r->n_q_heads, h->q_stride_token, h->q_stride_head) &&
              wide(h->k, r->n_k_heads, h->k_stride_token, h->k_stride_head);
    return PARASON_OK;
}

int check(const parason_rotate *r, pk::RotArgs *a)
{
    const int rc = check_sizes(r);
    if (rc != PARASON_OK) return rc;
    if ((r->dtype != PARASON_DTYPE_F32 && r->dtype != PARASON_DTYPE_BF16 && r->dtype != PARASON_DTYPE_F16) ||
        (r->flags & ~PARASON_ROTATE_INTERLEAVED) != 0 || !std::isfinite(r->eps) || !(r->eps > 0.0f))
        return PARASON_ERR_PARAM;
    if ((r->n_tokens > 0 && !r->positions) || (r->n_turned > 0 && !r->freqs)) return PARASON_ERR_NULL;
    const int64_t e = elem_of(r->dtype);
    if (!aligned(r->positions, 4) || !aligned(r->freqs, 8) || !aligned(r->q_weight, e) || !aligned(r->k_weight, e))
        return PARASON_ERR_ALIGN;
    a->n_tokens = r->n_tokens;
    a->q_heads = r->n_q_heads, a->k_heads = r->n_k_heads, a->dim = r->head_dim, a->half = r->n_turned / 2;
    a->group_log = 0;
    while ((16 << a->group_log) < a->dim) ++a->group_log;
    a->q_div = pk::fast_div((uint32_t)(a->q_heads > 0 ? a->q_heads : 1));
    a->k_div = pk::fast_div((uint32_t)(a->k_heads > 0 ? a->k_heads : 1));
    a->eps = r->eps, a->inv_dim = 1.0f / (float)a->dim;
    a->positions = r->positions, a->freqs = r->freqs;
    a->q_weight = (const char *)r->q_weight, a->k_weight = (const char *)r->k_weight;
    return PARASON_OK;
}

/* Tokens of a block at a time, at most as many as the block's table of angles holds.  Forward: as many as give each
 * thread an angle, but enough blocks.  Backward: all blocks get the same number, in as few rounds as that takes, but
 * at least a head for each group of lanes. */
int32_t tokens_at_once(const pk::RotArgs &a, bool grad)
{
    int64_t most = a.half > 0 ? pk::ROT_TURNS / a.half : pk::ROT_TOKENS;
    if (most > pk::ROT_TOKENS) most = pk::ROT_TOKENS;
    int64_t n = a.n_tokens / 1024;
    if (grad) {
        const int64_t blocks = pk::ROT_GRAD_BLOCKS, rounds = (a.n_tokens + blocks * most - 1) / (blocks * most);
        n = rounds > 0 ? (a.n_tokens + blocks * rounds - 1) / (blocks * rounds) : 1;
        const int64_t groups = pk::ROT_THREADS >> a.group_log, heads = a.q_heads + a.k_heads;
        if (n * heads < groups) n = heads > 0 ? (groups + heads - 1) / heads : most;
    } else if (a.half > 0 && most > (pk::ROT_THREADS + a.half - 1) / a.half) {
        most = (pk::ROT_THREADS + a.half - 1) / a.half;
    }
    if (n > most) n = most;
    return n > 1 ? (int32_t)n : 1;
}

int64_t grad_blocks(int64_t n_tokens) { return n_tokens < pk::ROT_GRAD_BLOCKS ? n_tokens : pk::ROT_GRAD_BLOCKS; }

RotKernel pick(const parason_rotate *r, bool grad)
{
    const bool inter = r->flags & PARASON_ROTATE_INTERLEAVED;
    return r->dtype == PARASON_DTYPE_F32    ? pick<PARASON_DTYPE_F32>(inter, grad)
           : r->dtype == PARASON_DTYPE_BF16 ? pick<PARASON_DTYPE_BF16>(inter, grad)
                                            : pick<PARASON_DTYPE_F16>(inter, grad);
}

}  // namespace

extern "C" {

int parason_qk_norm_rotate(const parason_rotate *r, const parason_heads *x, const parason_heads *y, void *stream)
{
    pk::RotArgs a = {};
    int rc = check(r, &a);
    if (rc == PARASON_OK) rc = check_heads(r, x, &a.x);
    if (rc == PARASON_OK) rc = check_heads(r, y, &a.y);
    if (rc != PARASON_OK) return rc;
    a.at_once = tokens_at_once(a, false);
    const int64_t blocks = (a.n_tokens + a.at_once - 1) / a.at_once;
    if (blocks > abi::MAX_BLOCKS) return PARASON_ERR_SIZE;
    if (blocks == 0 || a.q_heads + a.k_heads == 0) return PARASON_OK;
    if (abi::cu_count() <= 0) return PARASON_ERR_DEVICE;
    hipLaunchKernelGGL(pick(r, false), dim3((unsigned)blocks), dim3(pk::ROT_THREADS), 0, (hipStream_t)stream, a);
    return hipGetLastError() == hipSuccess ? PARASON_OK : PARASON_ERR_HIP;
}

int parason_qk_norm_rotate_workspace_size(const parason_rotate *r, size_t *bytes)
{
    if (!bytes) return PARASON_ERR_NULL;
    const int rc = check_sizes(r);
    if (rc != PARASON_OK) return rc;
    *bytes = abi::align_up((size_t)grad_blocks(r->n_tokens) * 2 * r->head_dim * sizeof(float) + 1);
    return PARASON_OK;
}

int parason_qk_norm_rotate_grad(const parason_rotate *r, const parason_heads *x, const parason_heads *dy, const parason_heads *dx,
                                float *q_weight_grad, float *k_weight_grad, void *workspace, size_t workspace_bytes, void *stream_ptr)
{
    pk::RotArgs a = {};
    int rc = check(r, &a);
    if (rc == PARASON_OK) rc = check_heads(r, x, &a.x);
    if (rc == PARASON_OK) rc = check_heads(r, dy, &a.g);
    if (rc == PARASON_OK) rc = check_heads(r, dx, &a.y);
    if (rc != PARASON_OK) return rc;
    if (!workspace) return PARASON_ERR_NULL;
    if (!aligned(q_weight_grad, 4) || !aligned(k_weight_grad, 4) || !aligned(workspace, abi::ALIGN)) return PARASON_ERR_ALIGN;
    size_t need;
    rc = parason_qk_norm_rotate_workspace_size(r, &need);
    if (rc != PARASON_OK) return rc;
    if (workspace_bytes < need) return PARASON_ERR_WORKSPACE;
    if (abi::cu_count() <= 0) return PARASON_ERR_DEVICE;
    a.sums = (float *)workspace;
    hipStream_t stream = (hipStream_t)stream_ptr;
    a.at_once = tokens_at_once(a, true);
    int64_t blocks = (a.n_tokens + a.at_once - 1) / a.at_once;
    blocks = blocks < grad_blocks(a.n_tokens) ? blocks : grad_blocks(a.n_tokens);
    if (blocks > 0) hipLaunchKernelGGL(pick(r, true), dim3((unsigned)blocks), dim3(pk::ROT_THREADS), 0, stream, a);
    if (q_weight_grad || k_weight_grad)
        hipLaunchKernelGGL(pk::rotate_weight_grad, dim3((unsigned)(2 * a.dim / 16)), dim3(pk::ROT_THREADS), 0, stream,
                           (const float *)workspace, (int32_t)blocks, a.dim, q_weight_grad, k_weight_grad);
    return hipGetLastError() == hipSuccess ? PARASON_OK : PARASON_ERR_HIP;
}

}  // extern "C"
