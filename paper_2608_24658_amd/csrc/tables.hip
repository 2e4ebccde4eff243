/*
 * tables.hip -- C-ABI of the cache's tables (kernels in tables_kernels.h).
 */
#include "kv_abi.h"
#include "tables_kernels.h"

using abi::align_up;
using abi::aligned;

namespace {

constexpr int64_t MAX_ROWS = 1 << 24;

struct TablesLayout {
    int64_t tiles;
    size_t tile_sums, off, end; /* the head at 0 */
};

TablesLayout layout_for(int64_t n)
{
    TablesLayout L;
    L.tiles = (n + pk::TABLE_TILE - 1) / pk::TABLE_TILE;
    L.tile_sums = align_up(2 * sizeof(int64_t));
    L.off = align_up(L.tile_sums + (size_t)L.tiles * 2 * sizeof(int64_t));
    L.end = align_up(L.off + (size_t)(n + 1) * sizeof(int64_t));
    return L;
}

int check(const parason_kv_pool *pool, const parason_kv_table *t, const int32_t *lengths, void *workspace, size_t workspace_bytes,
          pk::TableArgs *a)
{
    if (!pool || !t) return PARASON_ERR_NULL;
    if (t->n_rows < 0 || t->n_rows > MAX_ROWS || t->max_pages < 0 || t->page_size < 1 || pool->capacity < 0 ||
        pool->capacity > INT32_MAX || !abi::stride_fits(t->pages_stride, t->n_rows) ||
        (t->n_rows > 1 && t->pages_stride < t->max_pages))
        return PARASON_ERR_SIZE;
    if (!pool->free_count || (pool->capacity > 0 && !pool->free_pages) || !workspace ||
        (t->n_rows > 0 && (!t->kv_lens || !lengths || (t->max_pages > 0 && !t->pages))))
        return PARASON_ERR_NULL;
    if (!aligned(pool->free_pages, 4) || !aligned(pool->free_count, 4) || !aligned(t->kv_lens, 4) || !aligned(t->pages, 4) ||
        !aligned(lengths, 4) || !aligned(workspace, abi::ALIGN))
        return PARASON_ERR_ALIGN;
    const TablesLayout L = layout_for(t->n_rows);
    if (workspace_bytes < L.end) return PARASON_ERR_WORKSPACE;
    a->free_pages = pool->free_pages, a->free_count = pool->free_count, a->capacity = pool->capacity;
    a->n_rows = t->n_rows, a->kv_lens = t->kv_lens, a->pages = t->pages, a->pages_stride = t->pages_stride;
    a->max_pages = t->max_pages, a->page_size = t->page_size, a->page_div = pk::fast_div((uint32_t)t->page_size);
    a->most = (int64_t)t->max_pages * t->page_size;
    if (a->most > PARASON_KV_MAX_LEN) a->most = PARASON_KV_MAX_LEN;
    a->lengths = lengths;
    a->head = (int64_t *)workspace;
    a->tile_sums = (int64_t *)((char *)workspace + L.tile_sums);
    a->off = (int64_t *)((char *)workspace + L.off);
    return PARASON_OK;
}

}  // namespace

extern "C" {

int parason_kv_tables_workspace_size(int64_t n_rows, size_t *bytes)
{
    if (!bytes) return PARASON_ERR_NULL;
    if (n_rows < 0 || n_rows > MAX_ROWS) return PARASON_ERR_SIZE;
    *bytes = layout_for(n_rows).end;
    return PARASON_OK;
}

int parason_kv_extend(const parason_kv_pool *pool, const parason_kv_table *table, const int32_t *lengths, int64_t n_tokens,
                      const parason_kv_step *out, void *workspace, size_t workspace_bytes, void *stream_ptr)
{
    pk::TableArgs a = {};
    const int rc = check(pool, table, lengths, workspace, workspace_bytes, &a);
    if (rc != PARASON_OK) return rc;
    if (!out) return PARASON_ERR_NULL;
    if (n_tokens < 0 || n_tokens > INT32_MAX) return PARASON_ERR_SIZE;
    if (a.n_rows > 0 && (!out->lengths || !out->starts)) return PARASON_ERR_NULL;
    if (!aligned(out->lengths, 4) || !aligned(out->starts, 8) || !aligned(out->row_status, 4) || !aligned(out->positions, 4) ||
        !aligned(out->slots, 8) || !aligned(out->rows, 4))
        return PARASON_ERR_ALIGN;
    if (a.n_rows == 0 && n_tokens == 0) return PARASON_OK;
    if (abi::cu_count() <= 0) return PARASON_ERR_DEVICE;
    a.n_tokens = n_tokens;
    a.out_lengths = out->lengths, a.starts = out->starts, a.status = out->row_status;
    a.positions = out->positions, a.slots = out->slots, a.rows = out->rows;
    hipStream_t stream = (hipStream_t)stream_ptr;
    const dim3 threads(pk::TABLE_THREADS);
    if (a.n_rows <= pk::FEW_ROWS && n_tokens <= pk::FEW_TOKENS) {
        hipLaunchKernelGGL(pk::table_extend<true>, dim3(1), threads, 0, stream, a);
    } else {
        const int64_t tiles = layout_for(a.n_rows).tiles, blocks = (n_tokens + pk::FILL_TOKENS - 1) / pk::FILL_TOKENS;
        if (tiles > 1) hipLaunchKernelGGL(pk::table_sums<true>, dim3((unsigned)tiles), threads, 0, stream, a);
        if (tiles > 0) hipLaunchKernelGGL(pk::table_extend<false>, dim3((unsigned)tiles), threads, 0, stream, a);
        if (blocks > 0) hipLaunchKernelGGL(pk::table_fill, dim3((unsigned)blocks), dim3(pk::FILL_THREADS), 0, stream, a);
    }
    return hipGetLastError() == hipSuccess ? PARASON_OK : PARASON_ERR_HIP;
}

int parason_kv_shrink(const parason_kv_pool *pool, const parason_kv_table *table, const int32_t *new_lens, uint32_t *row_status,
                      void *workspace, size_t workspace_bytes, void *stream_ptr)
{
    pk::TableArgs a = {};
    const int rc = check(pool, table, new_lens, workspace, workspace_bytes, &a);
    if (rc != PARASON_OK) return rc;
    if (!aligned(row_status, 4)) return PARASON_ERR_ALIGN;
    if (a.n_rows == 0) return PARASON_OK;
    const int64_t pieces = (a.max_pages + pk::GIVE_PAGES - 1) / pk::GIVE_PAGES;
    const int64_t blocks = (a.n_rows * pieces + pk::FILL_THREADS / 64 - 1) / (pk::FILL_THREADS / 64);
    if (blocks > abi::MAX_BLOCKS) return PARASON_ERR_SIZE;
    if (abi::cu_count() <= 0) return PARASON_ERR_DEVICE;
    a.status = row_status;
    hipStream_t stream = (hipStream_t)stream_ptr;
    const dim3 threads(pk::TABLE_THREADS);
    if (a.n_rows <= pk::FEW_ROWS && a.n_rows * a.max_pages <= pk::FEW_PAGES) {
        hipLaunchKernelGGL(pk::table_shrink<true>, dim3(1), threads, 0, stream, a);
    } else {
        const int64_t tiles = layout_for(a.n_rows).tiles;
        if (tiles > 1) hipLaunchKernelGGL(pk::table_sums<false>, dim3((unsigned)tiles), threads, 0, stream, a);
        hipLaunchKernelGGL(pk::table_shrink<false>, dim3((unsigned)tiles), threads, 0, stream, a);
        if (blocks > 0) hipLaunchKernelGGL(pk::table_give, dim3((unsigned)blocks), dim3(pk::FILL_THREADS), 0, stream, a, pieces);
    }
    return hipGetLastError() == hipSuccess ? PARASON_OK : PARASON_ERR_HIP;
}

}  // extern "C"
