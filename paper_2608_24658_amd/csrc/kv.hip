/*
 * kv.hip -- C-ABI of the paged cache's write and read (kernels in
 * kv_kernels.h).
 */
#include "kv_abi.h"
#include "kv_kernels.h"

using abi::aligned;

namespace {

typedef void (*MoveKernel)(pk::KvMoveArgs);

template <template <int, int> class K>
MoveKernel pick(int dtype, int kind)
{
    constexpr int F32 = PARASON_DTYPE_F32, BF16 = PARASON_DTYPE_BF16, F16 = PARASON_DTYPE_F16;
    switch (kind) {
    case pk::KV_BF16: return dtype == F32 ? K<F32, pk::KV_BF16>::f : dtype == BF16 ? K<BF16, pk::KV_BF16>::f : K<F16, pk::KV_BF16>::f;
    case pk::KV_F16: return dtype == F32 ? K<F32, pk::KV_F16>::f : dtype == BF16 ? K<BF16, pk::KV_F16>::f : K<F16, pk::KV_F16>::f;
    case pk::KV_FP8: return dtype == F32 ? K<F32, pk::KV_FP8>::f : dtype == BF16 ? K<BF16, pk::KV_FP8>::f : K<F16, pk::KV_FP8>::f;
    default: return dtype == F32 ? K<F32, pk::KV_INT8>::f : dtype == BF16 ? K<BF16, pk::KV_INT8>::f : K<F16, pk::KV_INT8>::f;
    }
}

template <int T, int KIND>
struct Write {
    static constexpr MoveKernel f = pk::kv_write<T, KIND>;
};
template <int T, int KIND>
struct Read {
    static constexpr MoveKernel f = pk::kv_read<T, KIND>;
};

template <int T, int HEADS>
MoveKernel pick4(bool write)
{
    return write ? pk::kv_write4<T, HEADS> : pk::kv_read4<T, HEADS>;
}

template <int T>
MoveKernel pick4(bool write, int heads)
{
    return heads == 1 ? pick4<T, 1>(write) : heads == 2 ? pick4<T, 2>(write) : heads == pk::KV4_MORE ? pk::kv_read4<T, pk::KV4_MORE> : pick4<T, pk::KV4_HEADS>(write);
}

MoveKernel pick4(int dtype, bool write, int heads)
{
    return dtype == PARASON_DTYPE_F32    ? pick4<PARASON_DTYPE_F32>(write, heads)
           : dtype == PARASON_DTYPE_BF16 ? pick4<PARASON_DTYPE_BF16>(write, heads)
                                         : pick4<PARASON_DTYPE_F16>(write, heads);
}

/* Most blocks of a launch.  Rows are cut for the longest one, so many blocks of a ragged call find nothing to do, and
 * the few long rows need enough of theirs to fill the device: 48 rows of 1 to 36,000 positions, FP8 read as bfloat16,
 * 406 us at 8,192 blocks, 260 at 32,768, 267 at 131,072. */
constexpr int64_t MOVE_BLOCKS = 32768;

int move(const parason_kv_cache *cache, const parason_kv_rows *rows, const void *k, const void *v, int32_t dtype,
         int64_t stride_token, int64_t stride_head, uint32_t *row_status, void *stream_ptr, bool write)
{
    pk::KvMoveArgs a;
    int kind;
    int rc = abi::check_cache(cache, &a.c, &kind);
    if (rc != PARASON_OK) return rc;
    rc = abi::check_rows(rows, row_status, &a.r);
    if (rc != PARASON_OK) return rc;
    if (dtype != PARASON_DTYPE_F32 && dtype != PARASON_DTYPE_BF16 && dtype != PARASON_DTYPE_F16) return PARASON_ERR_PARAM;
    /* a 16-bit cache is written from its own type or from float32 */
    if (write && ((kind == pk::KV_BF16 && dtype == PARASON_DTYPE_F16) || (kind == pk::KV_F16 && dtype == PARASON_DTYPE_BF16)))
        return PARASON_ERR_PARAM;
    if (!abi::stride_fits(stride_token, rows->n_tokens) || !abi::stride_fits(stride_head, cache->n_heads)) return PARASON_ERR_SIZE;
    const int64_t elem = dtype == PARASON_DTYPE_F32 ? 4 : 2;
    /* units of a row (token, k or v, head) are counted in 31 bits */
    const int64_t units = (int64_t)rows->max_length * 2 * cache->n_heads;
    if (units > INT32_MAX || rows->n_rows > abi::MAX_BLOCKS) return PARASON_ERR_SIZE;
    if (rows->n_rows == 0 || rows->n_tokens == 0 || rows->max_length == 0) return PARASON_OK;
    if (!k || !v) return PARASON_ERR_NULL;
    if (!aligned(k, elem) || !aligned(v, elem)) return PARASON_ERR_ALIGN;
    if (abi::cu_count() <= 0) return PARASON_ERR_DEVICE;

    a.k = (char *)k, a.v = (char *)v;
    a.stride_token = stride_token, a.stride_head = stride_head;
    a.wide = aligned(k, 16) && aligned(v, 16) && stride_token * elem % 16 == 0 && stride_head * elem % 16 == 0;
    a.group = 1, a.group_log = 0;
    while (a.group * pk::KV_PER_LANE < cache->head_dim) a.group <<= 1, ++a.group_log;
    const bool four = kind == pk::KV_FP4;
    /* (only reads take KV4_MORE) */
    const int heads = !write && rows->n_tokens >= pk::KV4_MANY && cache->n_heads > pk::KV4_HEADS ? pk::KV4_MORE
                      : cache->n_heads < 3                                                       ? cache->n_heads
                                                                                                 : pk::KV4_HEADS;
    const int64_t chunks = four ? (cache->n_heads + heads - 1) / heads : cache->n_heads;
    a.heads_div = pk::fast_div((uint32_t)chunks);
    const int64_t per_block = pk::KV_THREADS / a.group * (four ? (heads < pk::KV4_HEADS ? pk::KV4_HEADS / heads : 1) : write ? pk::KV_WRITES : pk::KV_READS);
    int64_t blocks = (units / cache->n_heads * chunks + per_block - 1) / per_block, most = MOVE_BLOCKS / rows->n_rows;
    if (most < 1) most = 1; /* (as many blocks as rows) */
    if (blocks > most) blocks = most;
    a.blocks_per_row = (int32_t)blocks;
    const MoveKernel f = four ? pick4(dtype, write, heads) : write ? pick<Write>(dtype, kind) : pick<Read>(dtype, kind);
    hipLaunchKernelGGL(f, dim3((unsigned)(rows->n_rows * blocks)), dim3(pk::KV_THREADS), 0, (hipStream_t)stream_ptr, a);
    return hipGetLastError() == hipSuccess ? PARASON_OK : PARASON_ERR_HIP;
}

}  // namespace

extern "C" {

int parason_kv_write(const parason_kv_cache *cache, const parason_kv_rows *rows, const void *k, const void *v,
                     int32_t dtype, int64_t stride_token, int64_t stride_head, uint32_t *row_status, void *stream)
{
    return move(cache, rows, k, v, dtype, stride_token, stride_head, row_status, stream, true);
}

int parason_kv_read(const parason_kv_cache *cache, const parason_kv_rows *rows, void *k, void *v, int32_t dtype,
                    int64_t stride_token, int64_t stride_head, uint32_t *row_status, void *stream)
{
    return move(cache, rows, k, v, dtype, stride_token, stride_head, row_status, stream, false);
}

}  // extern "C"
