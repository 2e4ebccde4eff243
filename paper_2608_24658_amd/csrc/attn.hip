/*
 * attn.hip -- C-ABI of the attention of a tree of tokens over the paged cache
 * (kernels in attn_kernels.h).
 */
#include "kv_abi.h"
#include "attn_kernels.h"

using abi::aligned;
using abi::cu_count;

extern "C" {

int parason_tree_attention_workspace_size(const parason_kv_cache *cache, const parason_kv_rows *rows,
                                          int32_t n_q_heads, size_t *bytes)
{
    if (!bytes) return PARASON_ERR_NULL;
    pk::KvCache c;
    int kind;
    int rc = abi::check_cache(cache, &c, &kind);
    if (rc != PARASON_OK) return rc;
    rc = abi::check_row_sizes(rows);
    if (rc != PARASON_OK) return rc;
    if (n_q_heads < 1 || n_q_heads > PARASON_KV_MAX_HEADS || n_q_heads % cache->n_heads != 0) return PARASON_ERR_SIZE;
    *bytes = abi::ALIGN;
    return PARASON_OK;
}

int parason_tree_attention(const parason_kv_cache *cache, const parason_kv_rows *rows, const parason_tree_args *args,
                           uint32_t *row_status, void *workspace, size_t workspace_bytes, void *stream_ptr)
{
    if (!args) return PARASON_ERR_NULL;
    pk::TreeArgs a;
    int rc = abi::check_cache(cache, &a.c, &a.kind);
    if (rc != PARASON_OK) return rc;
    rc = abi::check_rows(rows, row_status, &a.r);
    if (rc != PARASON_OK) return rc;
    if (args->dtype != PARASON_DTYPE_BF16 && args->dtype != PARASON_DTYPE_F16) return PARASON_ERR_PARAM;
    if ((a.kind == pk::KV_BF16 && args->dtype != PARASON_DTYPE_BF16) ||
        (a.kind == pk::KV_F16 && args->dtype != PARASON_DTYPE_F16) || !std::isfinite(args->scale) ||
        (!args->mask && args->tree_lens))
        return PARASON_ERR_PARAM;
    size_t need;
    rc = parason_tree_attention_workspace_size(cache, rows, args->n_q_heads, &need);
    if (rc != PARASON_OK) return rc;
    if (!abi::stride_fits(args->q_stride_token, rows->n_tokens) || !abi::stride_fits(args->q_stride_head, args->n_q_heads) ||
        !abi::stride_fits(args->out_stride_token, rows->n_tokens) || !abi::stride_fits(args->out_stride_head, args->n_q_heads) ||
        (args->mask && (args->mask_words < 0 || !abi::stride_fits(args->mask_stride, rows->n_tokens))))
        return PARASON_ERR_SIZE;
    if (rows->n_rows == 0 || rows->n_tokens == 0 || rows->max_length == 0) return PARASON_OK;
    if (!args->q || !args->out || !workspace) return PARASON_ERR_NULL;
    if (!aligned(args->q, 2) || !aligned(args->out, 2) || !aligned(args->lse, 4) || !aligned(args->mask, 8) ||
        !aligned(args->tree_lens, 4) || !aligned(workspace, abi::ALIGN))
        return PARASON_ERR_ALIGN;
    if (workspace_bytes < need) return PARASON_ERR_WORKSPACE;
    if (cu_count() <= 0) return PARASON_ERR_DEVICE;

    a.q = (const char *)args->q, a.out = (char *)args->out, a.lse = args->lse;
    a.q_stride_token = args->q_stride_token, a.q_stride_head = args->q_stride_head;
    a.out_stride_token = args->out_stride_token, a.out_stride_head = args->out_stride_head;
    a.mask = args->mask, a.mask_stride = args->mask_stride, a.mask_words = args->mask_words;
    a.tree_lens = args->tree_lens;
    a.n_q_heads = args->n_q_heads;
    a.scale = args->scale;
    a.f16 = args->dtype == PARASON_DTYPE_F16;
    if (rows->n_rows > INT32_MAX / rows->max_length) return PARASON_ERR_SIZE;
    hipLaunchKernelGGL(pk::tree_attention_simple, dim3((unsigned)(rows->n_rows * rows->max_length), (unsigned)args->n_q_heads), dim3(256),
                       0, (hipStream_t)stream_ptr, a);
    return hipGetLastError() == hipSuccess ? PARASON_OK : PARASON_ERR_HIP;
}

}  // extern "C"
