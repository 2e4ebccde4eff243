/*
 * attn.hip -- C-ABI of the attention of a tree of tokens over the paged cache
 * (kernels in attn_kernels.h).
 */
#include "kv_abi.h"
#include "attn_kernels.h"

using abi::aligned;
using abi::cu_count;

namespace {

typedef void (*TreeKernel)(pk::TreeArgs);

template <int DP, int COLS>
TreeKernel pick_kind(bool f16, int kind)
{
    switch (kind) {
    case pk::KV_BF16: return pk::tree_attention<DP, COLS, false, pk::KV_BF16>;
    case pk::KV_F16: return pk::tree_attention<DP, COLS, true, pk::KV_F16>;
    case pk::KV_FP4: return f16 ? pk::tree_attention<DP, COLS, true, pk::KV_FP4> : pk::tree_attention<DP, COLS, false, pk::KV_FP4>;
    case pk::KV_FP8: return f16 ? pk::tree_attention<DP, COLS, true, pk::KV_FP8> : pk::tree_attention<DP, COLS, false, pk::KV_FP8>;
    default: return f16 ? pk::tree_attention<DP, COLS, true, pk::KV_INT8> : pk::tree_attention<DP, COLS, false, pk::KV_INT8>;
    }
}

template <int DP>
TreeKernel pick_cols(int cols, bool f16, int kind)
{
    return cols == 16 ? pick_kind<DP, 16>(f16, kind) : cols == 32 ? pick_kind<DP, 32>(f16, kind) : pick_kind<DP, 128>(f16, kind);
}

TreeKernel pick(int dim, int cols, bool f16, int kind)
{
    return dim <= 64 ? pick_cols<64>(cols, f16, kind) : dim <= 128 ? pick_cols<128>(cols, f16, kind) : pick_cols<256>(cols, f16, kind);
}

/* How a call is cut into blocks: by its sizes and bounds alone, so that the
 * workspace can be sized without a GPU. */
struct TreePlan {
    int32_t max_length; /* of the rows that can be good: their tokens are among the call's */
    int32_t cols, q_blocks, parts, part_len;
    int64_t rows;       /* of a launch; one does for all that are not many times the device's */
    size_t ml, end; /* workspace: the parts' vectors at 0, their maxima and sums at ml */
};

constexpr int64_t PART_BLOCKS = 1024;            /* blocks that a call is cut into */
constexpr size_t PART_BYTES = (size_t)1 << 29;   /* of the parts' vectors */

int plan(const parason_kv_cache *c, const parason_kv_rows *r, int32_t n_q_heads, TreePlan *p)
{
    const int64_t group = n_q_heads / c->n_heads;
    if (r->max_length * group > PARASON_KV_MAX_LEN) return PARASON_ERR_SIZE; /* (and blocks of columns end within 31 bits) */
    /* more than 2^31 blocks of 128 columns; the products below keep within 63 bits otherwise */
    if ((double)r->n_rows * r->max_length * n_q_heads > 0x1p38) return PARASON_ERR_SIZE;
    p->max_length = r->max_length < r->n_tokens ? r->max_length : (int32_t)r->n_tokens;
    const int64_t cols = p->max_length * group;
    p->cols = cols <= 16 ? 16 : cols <= 64 ? 32 : 128;
    p->q_blocks = cols == 0 ? 1 : (int32_t)((cols + p->cols - 1) / p->cols);
    /* blocks that have columns: those of a row's own tokens, at most one of them not full */
    int64_t base = r->n_rows * c->n_heads * p->q_blocks;
    const int64_t filled = (r->n_tokens * group / p->cols + r->n_rows) * c->n_heads;
    if (filled < base) base = filled;
    const int64_t tile = p->cols < 128 ? 128 : 64;
    /* Enough blocks to fill the device, and for few columns, whose partial results are small, parts short enough that
     * long rows among short ones do not finish last (4-bit positions are half as long as 8-bit ones, so that a part's
     * beginning and end weigh more: 128 single tokens 231 us in parts of 4,096, 278 in parts of 1,024).  A part is
     * worth its results: 8 bytes a column and value, written and read, against 2 to 4 bytes a position and value.  24
     * parts of prompts of 2 to 300 tokens behind 1 to 18,000 positions, all blocks the longest row would need counted:
     * 247 us, which is the longest row's; those with columns: 147. */
    const int64_t shortest = p->cols < 128 ? 512 : 1024;
    int64_t len = p->cols < 128 && c->dtype != PARASON_DTYPE_FP4 ? 1024 : 4096;
    while (len > shortest && base * ((r->max_kv_len + len - 1) / len) < PART_BLOCKS) len /= 2;
    const size_t per_part = (size_t)r->n_tokens * n_q_heads * c->head_dim * 4;
    int64_t parts = (r->max_kv_len + len - 1) / len;
    if (parts < 1 || base >= (p->cols < 128 ? 16 : 1) * PART_BLOCKS) parts = 1;
    if (per_part > 0 && (size_t)parts > PART_BYTES / per_part) parts = PART_BYTES / per_part > 1 ? (int64_t)(PART_BYTES / per_part) : 1;
    if (r->n_rows * p->max_length * n_q_heads > abi::MAX_BLOCKS * (pk::TREE_THREADS / 64)) parts = 1; /* tree_join's waves */
    len = (r->max_kv_len + parts - 1) / parts;
    p->part_len = (int32_t)((len + tile - 1) / tile * tile < INT32_MAX ? (len + tile - 1) / tile * tile : len);
    if (p->part_len < tile) p->part_len = (int32_t)tile;
    p->parts = (int32_t)parts;
    /* (their units rounded up to a multiple of eight) */
    p->rows = (abi::MAX_BLOCKS / p->q_blocks - 7) / (c->n_heads * parts);
    if (p->rows < 1) return PARASON_ERR_SIZE;
    p->ml = parts > 1 ? abi::align_up(per_part * parts) : 0;
    p->end = parts > 1 ? p->ml + abi::align_up((size_t)r->n_tokens * n_q_heads * 8 * parts) : abi::ALIGN;
    return PARASON_OK;
}

}  // namespace

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
    TreePlan p;
    rc = plan(cache, rows, n_q_heads, &p);
    if (rc == PARASON_OK) *bytes = p.end;
    return rc;
}

int parason_tree_attention(const parason_kv_cache *cache, const parason_kv_rows *rows, const parason_tree_args *args,
                           uint32_t *row_status, void *workspace, size_t workspace_bytes, void *stream_ptr)
{
    if (!args) return PARASON_ERR_NULL;
    pk::TreeArgs a;
    int kind;
    int rc = abi::check_cache(cache, &a.c, &kind);
    if (rc != PARASON_OK) return rc;
    rc = abi::check_rows(rows, row_status, &a.r);
    if (rc != PARASON_OK) return rc;
    if (args->dtype != PARASON_DTYPE_BF16 && args->dtype != PARASON_DTYPE_F16) return PARASON_ERR_PARAM;
    if ((kind == pk::KV_BF16 && args->dtype != PARASON_DTYPE_BF16) ||
        (kind == pk::KV_F16 && args->dtype != PARASON_DTYPE_F16) || !std::isfinite(args->scale) ||
        (!args->mask && args->tree_lens))
        return PARASON_ERR_PARAM;
    const int32_t heads = args->n_q_heads;
    if (heads < 1 || heads > PARASON_KV_MAX_HEADS || heads % cache->n_heads != 0) return PARASON_ERR_SIZE;
    if (!abi::stride_fits(args->q_stride_token, rows->n_tokens) || !abi::stride_fits(args->q_stride_head, heads) ||
        !abi::stride_fits(args->out_stride_token, rows->n_tokens) || !abi::stride_fits(args->out_stride_head, heads) ||
        (args->mask && (args->mask_words < 0 || !abi::stride_fits(args->mask_stride, rows->n_tokens))))
        return PARASON_ERR_SIZE;
    TreePlan p;
    rc = plan(cache, rows, heads, &p);
    if (rc != PARASON_OK) return rc;
    if (rows->n_rows == 0 || rows->n_tokens == 0 || rows->max_length == 0) return PARASON_OK;
    if (!args->q || !args->out || !workspace) return PARASON_ERR_NULL;
    if (!aligned(args->q, 2) || !aligned(args->out, 2) || !aligned(args->lse, 4) || !aligned(args->mask, 8) ||
        !aligned(args->tree_lens, 4) || !aligned(workspace, abi::ALIGN))
        return PARASON_ERR_ALIGN;
    if (workspace_bytes < p.end) return PARASON_ERR_WORKSPACE;
    if (cu_count() <= 0) return PARASON_ERR_DEVICE;

    a.q = (const char *)args->q, a.out = (char *)args->out, a.lse = args->lse;
    a.q_stride_token = args->q_stride_token, a.q_stride_head = args->q_stride_head;
    a.out_stride_token = args->out_stride_token, a.out_stride_head = args->out_stride_head;
    a.q_wide = aligned(args->q, 16) && args->q_stride_token % 8 == 0 && args->q_stride_head % 8 == 0;
    a.out_wide = aligned(args->out, 8) && args->out_stride_token % 4 == 0 && args->out_stride_head % 4 == 0;
    a.mask = args->mask, a.mask_stride = args->mask_stride, a.mask_words = args->mask_words;
    a.tree_lens = args->tree_lens;
    a.n_q_heads = heads;
    a.group = heads / cache->n_heads;
    a.group_div = pk::fast_div((uint32_t)a.group);
    a.negate = args->scale < 0.0f;
    const float c2 = (float)(std::fabs((double)args->scale) * 1.4426950408889634);
    a.c2 = c2 > 0x1p-126f ? c2 : 0x1p-126f;
    a.q_blocks = p.q_blocks, a.parts = p.parts, a.part_len = p.part_len;
    a.q_blocks_div = pk::fast_div((uint32_t)p.q_blocks), a.parts_div = pk::fast_div((uint32_t)p.parts);
    a.heads_div = pk::fast_div((uint32_t)cache->n_heads), a.part_len_div = pk::fast_div((uint32_t)p.part_len);
    a.r.max_length = p.max_length;
    a.part_out = (float *)workspace;
    a.part_ml = (float2 *)((char *)workspace + p.ml);
    const bool f16 = args->dtype == PARASON_DTYPE_F16;
    hipStream_t stream = (hipStream_t)stream_ptr;
    const TreeKernel f = pick(cache->head_dim, p.cols, f16, kind);
    for (int64_t i = 0; i < rows->n_rows; i += p.rows) {
        pk::TreeArgs b = a;
        b.r.n_rows = rows->n_rows - i < p.rows ? rows->n_rows - i : p.rows;
        b.r.starts += i, b.r.lengths += i, b.r.kv_lens += i;
        if (b.r.pages) b.r.pages += i * b.r.pages_stride;
        if (b.r.status) b.r.status += i;
        if (b.tree_lens) b.tree_lens += i;
        b.units = (uint32_t)(b.r.n_rows * cache->n_heads * p.parts);
        b.by_xcd = p.q_blocks > 1 && b.units >= 8;
        const int64_t blocks = (int64_t)(b.by_xcd ? (b.units + 7) / 8 * 8 : b.units) * p.q_blocks;
        hipLaunchKernelGGL(f, dim3((unsigned)blocks), dim3(pk::TREE_THREADS), 0, stream, b);
    }
    if (p.parts > 1) {
        constexpr int64_t per_block = pk::TREE_THREADS / 64;
        /* (2^26 waves at most, and so many tokens and heads of a row) */
        const int64_t waves = rows->n_rows * p.max_length * heads;
        a.row_div = pk::fast_div((uint32_t)(p.max_length * heads)), a.q_heads_div = pk::fast_div((uint32_t)heads);
        hipLaunchKernelGGL(f16 ? pk::tree_join<true> : pk::tree_join<false>, dim3((unsigned)((waves + per_block - 1) / per_block)),
                           dim3(pk::TREE_THREADS), 0, stream, a, p.cols);
    }
    return hipGetLastError() == hipSuccess ? PARASON_OK : PARASON_ERR_HIP;
}

}  // extern "C"
