/*
 * beam.hip -- C-ABI of the beam selection and reordering (kernels in
 * beam_kernels.h).
 */
#include "kv_abi.h"
#include "beam_kernels.h"

using abi::aligned;
using abi::cu_count;

namespace {

struct BeamLayout {
    int64_t chunks;
    size_t best, end; /* the chunks' sums at 0 */
};

int layout_for(int64_t n_groups, int32_t beams, int64_t vocab, BeamLayout *L)
{
    if (n_groups < 0 || beams < 1 || beams > PARASON_BEAM_MAX || n_groups > INT32_MAX / beams || vocab < 1 || vocab > INT32_MAX - 1)
        return PARASON_ERR_SIZE;
    L->chunks = (vocab + pk::BEAM_CHUNK - 1) / pk::BEAM_CHUNK;
    const int64_t rows = n_groups * beams;
    if (rows > abi::MAX_BLOCKS / L->chunks) return PARASON_ERR_SIZE;
    L->best = abi::align_up((size_t)(rows * L->chunks) * sizeof(pk::BeamChunk));
    L->end = L->best + abi::align_up((size_t)(rows * L->chunks) * beams * sizeof(pk::BeamCandidate) + 1);
    return PARASON_OK;
}

struct Rows {
    const char *p;
    int64_t bytes, stride; /* 0 < bytes <= stride */
};

/* Whether any of n rows here and n rows there share a byte. */
bool rows_meet(const Rows &a, const Rows &b, int64_t n)
{
    const int64_t d = (int64_t)((uintptr_t)b.p - (uintptr_t)a.p); /* rows of b from the first byte of a on */
    if (d >= (n - 1) * a.stride + a.bytes || -d >= (n - 1) * b.stride + b.bytes) return false;
    if (a.stride == b.stride) { /* as far behind a row of a, or between two, as all of them */
        const int64_t in = (d % a.stride + a.stride) % a.stride;
        return in < a.bytes || in + b.bytes > a.stride;
    }
    for (int64_t i = 0, j = 0; i < n && j < n;) {
        const int64_t x = i * a.stride, y = d + j * b.stride;
        if (x + a.bytes <= y) i += (y - x - a.bytes) / a.stride + 1;      /* the first that ends behind y */
        else if (y + b.bytes <= x) j += (x - y - b.bytes) / b.stride + 1;
        else return true;
    }
    return false;
}

}  // namespace

extern "C" {

int parason_beam_workspace_size(int64_t n_groups, int32_t beams, int64_t vocab, size_t *bytes)
{
    if (!bytes) return PARASON_ERR_NULL;
    BeamLayout L;
    const int rc = layout_for(n_groups, beams, vocab, &L);
    if (rc == PARASON_OK) *bytes = L.end;
    return rc;
}

int parason_beam_select(const void *logits, int64_t vocab, int64_t row_stride, int32_t dtype, const float *scores,
                        const parason_decode_state *states, int64_t n_groups, int32_t beams, float *new_scores,
                        int32_t *parents, int32_t *tokens, void *workspace, size_t workspace_bytes, void *stream_ptr)
{
    BeamLayout L;
    const int rc = layout_for(n_groups, beams, vocab, &L);
    if (rc != PARASON_OK) return rc;
    const int64_t rows = n_groups * beams;
    if (row_stride < vocab || row_stride > INT64_MAX / 8 / (rows > 0 ? rows : 1)) return PARASON_ERR_SIZE;
    if (dtype != PARASON_DTYPE_F32 && dtype != PARASON_DTYPE_BF16 && dtype != PARASON_DTYPE_F16) return PARASON_ERR_PARAM;
    if (rows == 0) return PARASON_OK;
    if (!logits || !scores || !new_scores || !parents || !tokens || !workspace) return PARASON_ERR_NULL;
    const int64_t elem = dtype == PARASON_DTYPE_F32 ? 4 : 2;
    if (!aligned(logits, elem) || !aligned(scores, 4) || !aligned(states, 16) || !aligned(new_scores, 4) ||
        !aligned(parents, 4) || !aligned(tokens, 4) || !aligned(workspace, abi::ALIGN))
        return PARASON_ERR_ALIGN;
    if (workspace_bytes < L.end) return PARASON_ERR_WORKSPACE;
    if (cu_count() <= 0) return PARASON_ERR_DEVICE;
    pk::BeamArgs a;
    a.logits = (const char *)logits;
    a.vocab = vocab, a.row_bytes = row_stride * elem, a.dtype = dtype;
    a.scores = scores, a.states = states, a.beams = beams, a.chunks = (int32_t)L.chunks;
    a.chunks_div = pk::fast_div((uint32_t)L.chunks);
    const int64_t pieces = (vocab * elem + 15) / 16;
    a.chunk_pieces = (int32_t)((pieces + L.chunks - 1) / L.chunks);
    a.chunk_tokens = (int64_t)a.chunk_pieces * (16 / elem);
    a.sums = (pk::BeamChunk *)workspace;
    a.best = (pk::BeamCandidate *)((char *)workspace + L.best);
    a.new_scores = new_scores, a.parents = parents, a.tokens = tokens;
    hipStream_t stream = (hipStream_t)stream_ptr;
    auto scan = dtype == PARASON_DTYPE_F32 ? pk::beam_scan<PARASON_DTYPE_F32>
                : dtype == PARASON_DTYPE_BF16 ? pk::beam_scan<PARASON_DTYPE_BF16> : pk::beam_scan<PARASON_DTYPE_F16>;
    hipLaunchKernelGGL(scan, dim3((unsigned)(rows * L.chunks)), dim3(pk::BEAM_THREADS), 0, stream, a);
    hipLaunchKernelGGL(pk::beam_choose, dim3((unsigned)n_groups), dim3(pk::BEAM_THREADS), 0, stream, a);
    return hipGetLastError() == hipSuccess ? PARASON_OK : PARASON_ERR_HIP;
}

int parason_beam_reorder(const int32_t *parents, int64_t n_rows, const parason_beam_array *arrays, int32_t n_arrays,
                         void *stream_ptr)
{
    if (n_rows < 0 || n_rows > abi::MAX_BLOCKS || n_arrays < 0 || n_arrays > PARASON_BEAM_ARRAYS) return PARASON_ERR_SIZE;
    if (n_rows == 0 || n_arrays == 0) return PARASON_OK;
    if (!parents || !arrays) return PARASON_ERR_NULL;
    pk::ReorderArgs a;
    a.parents = parents, a.n_rows = n_rows, a.n_arrays = 0;
    int64_t blocks = 0;
    for (int small = 1; small >= 0; --small) {
        if (!small) {
            a.n_small = a.n_arrays;
            blocks = a.n_small > 0; /* block 0 of a row: the small arrays */
        }
        for (int k = 0; k < n_arrays; ++k) {
            const parason_beam_array &x = arrays[k];
            if (x.row_bytes < 0 || x.src_stride < x.row_bytes || x.dst_stride < x.row_bytes ||
                !abi::stride_fits(x.src_stride, n_rows) || !abi::stride_fits(x.dst_stride, n_rows))
                return PARASON_ERR_SIZE;
            if (x.row_bytes == 0 || (x.row_bytes <= pk::REORDER_SMALL) != (small == 1)) continue;
            if (!x.src || !x.dst) return PARASON_ERR_NULL;
            const uintptr_t ends = (uintptr_t)x.src | (uintptr_t)x.dst | (uintptr_t)x.src_stride | (uintptr_t)x.dst_stride;
            a.width[a.n_arrays] = (ends & 15u) == 0 ? 16 : (ends & 3u) == 0 ? 4 : 1;
            a.first_block[a.n_arrays] = (int32_t)blocks;
            a.arrays[a.n_arrays++] = x;
            if (!small) blocks += (x.row_bytes + pk::REORDER_SEGMENT - 1) / pk::REORDER_SEGMENT;
            if (blocks > abi::MAX_BLOCKS / n_rows) return PARASON_ERR_SIZE;
        }
    }
    if (!aligned(parents, 4)) return PARASON_ERR_ALIGN;
    if (a.n_arrays == 0) return PARASON_OK;
    for (int k = 0; k < a.n_arrays; ++k) { /* rows are written while others are read */
        const parason_beam_array &x = a.arrays[k];
        const Rows dst{(const char *)x.dst, x.row_bytes, x.dst_stride};
        if (rows_meet(dst, Rows{(const char *)parents, 4, 4}, n_rows)) return PARASON_ERR_PARAM;
        for (int m = 0; m < a.n_arrays; ++m) {
            const parason_beam_array &y = a.arrays[m];
            if (rows_meet(dst, Rows{(const char *)y.src, y.row_bytes, y.src_stride}, n_rows) ||
                (m < k && rows_meet(dst, Rows{(const char *)y.dst, y.row_bytes, y.dst_stride}, n_rows)))
                return PARASON_ERR_PARAM;
        }
    }
    if (cu_count() <= 0) return PARASON_ERR_DEVICE;
    a.blocks_per_row = (int32_t)blocks;
    hipLaunchKernelGGL(pk::beam_reorder, dim3((unsigned)(n_rows * blocks)), dim3(pk::REORDER_THREADS), 0, (hipStream_t)stream_ptr, a);
    return hipGetLastError() == hipSuccess ? PARASON_OK : PARASON_ERR_HIP;
}

}  // extern "C"
