/*
 * beam.hip -- C-ABI of the beam selection and reordering (kernels in
 * beam_kernels.h).
 */
#include "kv_abi.h"
#include "beam_kernels.h"

using abi::aligned;
using abi::cu_count;

namespace {

int check_sizes(int64_t n_groups, int32_t beams, int64_t vocab)
{
    if (n_groups < 0 || beams < 1 || beams > PARASON_BEAM_MAX || n_groups > INT32_MAX / beams || vocab < 1 || vocab > INT32_MAX - 1)
        return PARASON_ERR_SIZE;
    return PARASON_OK;
}

}  // namespace

extern "C" {

int parason_beam_workspace_size(int64_t n_groups, int32_t beams, int64_t vocab, size_t *bytes)
{
    if (!bytes) return PARASON_ERR_NULL;
    const int rc = check_sizes(n_groups, beams, vocab);
    if (rc != PARASON_OK) return rc;
    *bytes = abi::align_up((size_t)(n_groups * beams) * 8 + 1);
    return PARASON_OK;
}

int parason_beam_select(const void *logits, int64_t vocab, int64_t row_stride, int32_t dtype, const float *scores,
                        const parason_decode_state *states, int64_t n_groups, int32_t beams, float *new_scores,
                        int32_t *parents, int32_t *tokens, void *workspace, size_t workspace_bytes, void *stream_ptr)
{
    size_t need;
    const int rc = parason_beam_workspace_size(n_groups, beams, vocab, &need);
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
    if (workspace_bytes < need) return PARASON_ERR_WORKSPACE;
    if (cu_count() <= 0) return PARASON_ERR_DEVICE;
    pk::BeamArgs a;
    a.logits = (const char *)logits;
    a.vocab = vocab, a.row_bytes = row_stride * elem, a.rows = rows;
    a.scores = scores, a.states = states, a.beams = beams;
    a.norm = (double *)workspace;
    a.new_scores = new_scores, a.parents = parents, a.tokens = tokens;
    hipStream_t stream = (hipStream_t)stream_ptr;
    auto norm = dtype == PARASON_DTYPE_F32 ? pk::beam_norm<PARASON_DTYPE_F32>
                : dtype == PARASON_DTYPE_BF16 ? pk::beam_norm<PARASON_DTYPE_BF16> : pk::beam_norm<PARASON_DTYPE_F16>;
    auto rounds = dtype == PARASON_DTYPE_F32 ? pk::beam_rounds<PARASON_DTYPE_F32>
                  : dtype == PARASON_DTYPE_BF16 ? pk::beam_rounds<PARASON_DTYPE_BF16> : pk::beam_rounds<PARASON_DTYPE_F16>;
    hipLaunchKernelGGL(norm, dim3((unsigned)rows), dim3(pk::BEAM_THREADS), 0, stream, a);
    hipLaunchKernelGGL(rounds, dim3((unsigned)n_groups), dim3(pk::BEAM_THREADS), 0, stream, a);
    return hipGetLastError() == hipSuccess ? PARASON_OK : PARASON_ERR_HIP;
}

int parason_beam_reorder(const int32_t *parents, int64_t n_rows, const parason_beam_array *arrays, int32_t n_arrays,
                         void *stream_ptr)
{
    if (n_rows < 0 || n_rows > INT32_MAX || n_arrays < 0 || n_arrays > PARASON_BEAM_ARRAYS) return PARASON_ERR_SIZE;
    if (n_rows == 0 || n_arrays == 0) return PARASON_OK;
    if (!parents || !arrays) return PARASON_ERR_NULL;
    pk::ReorderArgs a;
    a.parents = parents, a.n_rows = n_rows, a.n_arrays = 0;
    for (int k = 0; k < n_arrays; ++k) {
        const parason_beam_array &x = arrays[k];
        if (x.row_bytes < 0 || x.src_stride < x.row_bytes || x.dst_stride < x.row_bytes ||
            !abi::stride_fits(x.src_stride, n_rows) || !abi::stride_fits(x.dst_stride, n_rows))
            return PARASON_ERR_SIZE;
        if (x.row_bytes == 0) continue;
        if (!x.src || !x.dst) return PARASON_ERR_NULL;
        a.arrays[a.n_arrays++] = x;
    }
    if (!aligned(parents, 4)) return PARASON_ERR_ALIGN;
    if (a.n_arrays == 0) return PARASON_OK;
    if (cu_count() <= 0) return PARASON_ERR_DEVICE;
    hipLaunchKernelGGL(pk::beam_reorder, dim3((unsigned)n_rows), dim3(256), 0, (hipStream_t)stream_ptr, a);
    return hipGetLastError() == hipSuccess ? PARASON_OK : PARASON_ERR_HIP;
}

}  // extern "C"
