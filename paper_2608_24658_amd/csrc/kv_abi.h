/*
 * kv_abi.h -- host checks of the cache and of a call's rows, shared by the
 * entry points that take them.
 */
#pragma once
#include "abi_common.h"
#include "kv_common.h"

namespace abi {

constexpr int64_t MAX_ELEMS = (int64_t)1 << 56; /* no product of a stride and an index overflows below this */

/* Blocks of 256 threads that a launch takes: a grid of 2^32 threads or more is refused or, worse, cut to 32 bits. */
constexpr int64_t MAX_BLOCKS = 0xFFFFFFFFll / 256;

inline bool aligned(const void *p, size_t n) { return ((uintptr_t)p & (n - 1)) == 0; }

/* |stride| * count stays within MAX_ELEMS */
inline bool stride_fits(int64_t stride, int64_t count)
{
    return count <= 0 || (stride <= MAX_ELEMS / count && stride >= -(MAX_ELEMS / count));
}

/* Check a cache's description and fill in the kernels' view of it. */
inline int check_cache(const parason_kv_cache *c, pk::KvCache *o, int *kind)
{
    if (!c) return PARASON_ERR_NULL;
    switch (c->dtype) {
    case PARASON_DTYPE_BF16: *kind = pk::KV_BF16; break;
    case PARASON_DTYPE_F16: *kind = pk::KV_F16; break;
    case PARASON_DTYPE_FP8: *kind = pk::KV_FP8; break;
    case PARASON_DTYPE_INT8: *kind = pk::KV_INT8; break;
    case PARASON_DTYPE_FP4: *kind = pk::KV_FP4; break;
    default: return PARASON_ERR_PARAM;
    }
    const bool four = *kind == pk::KV_FP4, codes = *kind == pk::KV_FP8 || *kind == pk::KV_INT8 || four;
    if (c->n_pages < 0 || c->n_pages > INT32_MAX || c->page_size < 1 || c->n_heads < 1 ||
        c->n_heads > PARASON_KV_MAX_HEADS || c->head_dim < 16 || c->head_dim > PARASON_KV_MAX_DIM ||
        c->head_dim % (four ? PARASON_KV_SCALE_GROUP : 16) != 0)
        return PARASON_ERR_SIZE;
    if (!stride_fits(c->stride_page, c->n_pages) || !stride_fits(c->stride_slot, c->page_size) ||
        !stride_fits(c->stride_head, c->n_heads) ||
        (codes && (!stride_fits(c->scale_stride_page, c->n_pages) ||
                   !stride_fits(c->scale_stride_slot, c->page_size) ||
                   !stride_fits(c->scale_stride_head, c->n_heads))))
        return PARASON_ERR_SIZE;
    if (c->n_pages > 0 && (!c->k || !c->v || (codes && (!c->k_scale || !c->v_scale)))) return PARASON_ERR_NULL;
    const int64_t unit = four ? 32 : codes ? 16 : 8; /* elements of 16 bytes */
    if (!aligned(c->k, 16) || !aligned(c->v, 16) || c->stride_page % unit != 0 || c->stride_slot % unit != 0 ||
        c->stride_head % unit != 0 || (codes && !four && (!aligned(c->k_scale, 4) || !aligned(c->v_scale, 4))))
        return PARASON_ERR_ALIGN;
    o->k = (char *)c->k;
    o->v = (char *)c->v;
    o->k_scale = codes ? (float *)c->k_scale : nullptr;
    o->v_scale = codes ? (float *)c->v_scale : nullptr;
    o->n_pages = c->n_pages;
    o->stride_page = c->stride_page, o->stride_slot = c->stride_slot, o->stride_head = c->stride_head;
    o->scale_stride_page = c->scale_stride_page, o->scale_stride_slot = c->scale_stride_slot;
    o->scale_stride_head = c->scale_stride_head;
    o->page_size = c->page_size, o->n_heads = c->n_heads, o->head_dim = c->head_dim;
    o->page_div = pk::fast_div((uint32_t)c->page_size);
    return PARASON_OK;
}

/* Sizes of the rows alone (what a workspace is sized by). */
inline int check_row_sizes(const parason_kv_rows *r)
{
    if (!r) return PARASON_ERR_NULL;
    if (r->n_rows < 0 || r->n_rows > INT32_MAX || r->n_tokens < 0 || r->n_tokens > INT32_MAX || r->max_pages < 0 ||
        r->max_length < 0 || r->max_kv_len < 0 || r->max_kv_len > PARASON_KV_MAX_LEN ||
        !stride_fits(r->pages_stride, r->n_rows))
        return PARASON_ERR_SIZE;
    return PARASON_OK;
}

inline int check_rows(const parason_kv_rows *r, uint32_t *status, pk::KvRows *o)
{
    const int rc = check_row_sizes(r);
    if (rc != PARASON_OK) return rc;
    if (r->n_rows > 0 && (!r->starts || !r->lengths || !r->kv_lens || (r->max_pages > 0 && !r->pages)))
        return PARASON_ERR_NULL;
    if (!aligned(r->starts, 8) || !aligned(r->lengths, 4) || !aligned(r->kv_lens, 4) || !aligned(r->pages, 4) ||
        !aligned(status, 4))
        return PARASON_ERR_ALIGN;
    o->n_rows = r->n_rows, o->n_tokens = r->n_tokens;
    o->starts = r->starts, o->lengths = r->lengths, o->kv_lens = r->kv_lens, o->pages = r->pages;
    o->pages_stride = r->pages_stride;
    o->max_pages = r->max_pages, o->max_length = r->max_length, o->max_kv_len = r->max_kv_len;
    o->status = status;
    return PARASON_OK;
}

}  // namespace abi
