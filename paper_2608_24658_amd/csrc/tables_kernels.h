/*
 * tables_kernels.h -- the cache's tables on gfx950: pages taken for new
 * positions and given back, and where every new token belongs.
 *
 * Both directions are an exclusive sum over the rows (of the new tokens and of
 * the pages that move) and then independent work for each token or page.  The
 * sums are one block's over TABLE_TILE rows; more rows take a launch before it
 * that sums each tile.  The work of each token finds its row by a search in the
 * sums, so that a long prompt among single tokens is spread like the others.
 */
#pragma once
#include "kv_common.h"

namespace pk {

constexpr int TABLE_THREADS = 1024, TABLE_PER = 4;          /* rows of a thread */
constexpr int TABLE_TILE = TABLE_THREADS * TABLE_PER;
constexpr int FILL_THREADS = 256, FILL_PER = 4;             /* tokens of a thread */
constexpr int FILL_TOKENS = FILL_THREADS * FILL_PER;
constexpr int GIVE_PAGES = 512;                             /* pages of a row that one wave gives back */

struct TableArgs {
    int32_t *free_pages, *free_count;
    int64_t capacity;
    int64_t n_rows;
    int32_t *kv_lens, *pages;
    int64_t pages_stride;
    int32_t max_pages, page_size;
    FastDiv page_div;
    int64_t most;                /* positions that a row may have */
    const int32_t *lengths;      /* extend: new tokens; shrink: positions that stay */
    int64_t n_tokens;
    int32_t *out_lengths;
    int64_t *starts;
    int32_t *positions, *rows;
    int64_t *slots;
    uint32_t *status;
    int64_t *tile_sums;          /* [tiles][2]: tokens, pages (several tiles) */
    int64_t *off;                /* [n_rows + 1]: pages that move before the row's */
    int64_t *head;               /* [1]: free pages before the call, [1]: pages that move */
};

__device__ __forceinline__ int64_t wave_upto(int64_t x)
{
    const int lane = (int)threadIdx.x & 63;
#pragma unroll
    for (int k = 1; k < 64; k <<= 1) {
        const int64_t y = __shfl_up(x, k);
        if (lane >= k) x += y;
    }
    return x;
}

/* Sum over the block, and of the threads before this one. */
__device__ __forceinline__ int64_t block_before(int64_t x, int64_t *lds, int64_t *total)
{
    const int wave = (int)threadIdx.x >> 6, waves = (int)blockDim.x >> 6;
    const int64_t upto = wave_upto(x);
    if ((threadIdx.x & 63) == 63) lds[wave] = upto;
    __syncthreads();
    int64_t before = upto - x, sum = 0;
    for (int i = 0; i < waves; ++i) {
        const int64_t s = lds[i];
        before += i < wave ? s : 0;
        sum += s;
    }
    __syncthreads();
    *total = sum;
    return before;
}

__device__ __forceinline__ int32_t pages_for(const TableArgs &a, int32_t n)
{
    const uint32_t q = div_by((uint32_t)n, a.page_div);
    return (int32_t)(q + (q * (uint32_t)a.page_size < (uint32_t)n));
}

__device__ __forceinline__ int64_t free_pages_of(const TableArgs &a)
{
    const int64_t n = *a.free_count;
    return n < 0 ? 0 : n < a.capacity ? n : a.capacity;
}

/* What a row asks for, whatever the others do. */
struct TableRow {
    int32_t old, n;      /* positions before; extend: new tokens, shrink: positions that stay */
    int32_t pages;       /* that move */
    bool good;
};

template <bool EXTEND>
__device__ __forceinline__ TableRow table_row(const TableArgs &a, int64_t i)
{
    TableRow r = {0, 0, 0, false};
    if (i >= a.n_rows) return r;
    r.old = a.kv_lens[i];
    r.n = a.lengths[i];
    if (EXTEND) {
        r.good = r.n >= 0 && r.old >= 0 && (int64_t)r.old + r.n <= a.most;
        if (r.good) r.pages = pages_for(a, r.old + r.n) - pages_for(a, r.old);
    } else {
        r.good = r.n >= 0 && r.n <= r.old && r.old <= a.most;
        if (r.good) r.pages = pages_for(a, r.old) - pages_for(a, r.n);
    }
    return r;
}

/* The sums of a tile of rows. */
template <bool EXTEND>
__global__ void __launch_bounds__(TABLE_THREADS) table_sums(TableArgs a)
{
    __shared__ int64_t lds[TABLE_THREADS / 64];
    int64_t tokens = 0, pages = 0;
    for (int k = 0; k < TABLE_PER; ++k) {
        const TableRow r = table_row<EXTEND>(a, (int64_t)blockIdx.x * TABLE_TILE + k * TABLE_THREADS + threadIdx.x);
        tokens += r.n > 0 ? r.n : 0;
        pages += r.pages;
    }
    int64_t sum;
    block_before(tokens, lds, &sum);
    if (threadIdx.x == 0) a.tile_sums[2 * blockIdx.x] = sum;
    block_before(pages, lds, &sum);
    if (threadIdx.x == 0) a.tile_sums[2 * blockIdx.x + 1] = sum;
    if (blockIdx.x == 0 && threadIdx.x == 0) a.head[0] = free_pages_of(a);
}

/* One token of row `row`: where it goes, and the table's entry where it is its page's first. */
__device__ __forceinline__ void place_token(const TableArgs &a, int64_t t, bool served, int64_t row, int64_t at_in_row, int32_t old,
                                            int64_t off, int64_t free_before)
{
    int32_t at = -1;
    int64_t slot = -1;
    if (served) {
        at = old + (int32_t)at_in_row;
        const int32_t nth = (int32_t)div_by((uint32_t)at, a.page_div), in = at - nth * a.page_size, had = pages_for(a, old);
        int32_t *const entry = a.pages + row * a.pages_stride + nth;
        int32_t page;
        if (nth >= had) {
            page = a.free_pages[free_before - 1 - (off + nth - had)];
            if (in == 0) *entry = page;
        } else {
            page = *entry;
        }
        if (page >= 0) slot = (int64_t)page * a.page_size + in;
    }
    if (a.positions) a.positions[t] = at;
    if (a.slots) a.slots[t] = slot;
    if (a.rows) a.rows[t] = served ? (int32_t)row : -1;
}

/* Sums over the rows, and what a row keeps of them.  FEW (one row a thread, few
 * tokens or pages): what follows is done by the same block. */
constexpr int FEW_ROWS = TABLE_THREADS, FEW_TOKENS = 4 * TABLE_THREADS;
constexpr int64_t FEW_PAGES = 64 * TABLE_THREADS;

template <bool FEW>
__global__ void __launch_bounds__(TABLE_THREADS) table_extend(TableArgs a)
{
    constexpr int PER = FEW ? 1 : TABLE_PER;
    __shared__ int64_t lds[TABLE_THREADS / 64];
    __shared__ int32_t first[FEW ? FEW_ROWS : 1], olds[FEW ? FEW_ROWS : 1], offs[FEW ? FEW_ROWS : 1], taken[FEW ? FEW_ROWS : 1];
    const int tid = (int)threadIdx.x;
    const int64_t row0 = (int64_t)blockIdx.x * TABLE_THREADS * PER + tid * PER;
    const bool one = gridDim.x == 1;
    int64_t tokens_before = 0, pages_before = 0;
    if (!one) {
        int64_t t = 0, p = 0;
        for (int64_t i = tid; i < blockIdx.x; i += TABLE_THREADS) t += a.tile_sums[2 * i], p += a.tile_sums[2 * i + 1];
        block_before(t, lds, &tokens_before);
        block_before(p, lds, &pages_before);
    }
    const int64_t have = one ? free_pages_of(a) : a.head[0];
    TableRow r[PER];
    int64_t tokens = 0, pages = 0;
#pragma unroll
    for (int k = 0; k < PER; ++k) {
        r[k] = table_row<true>(a, row0 + k);
        tokens += r[k].n > 0 ? r[k].n : 0;
        pages += r[k].pages;
    }
    int64_t sum, total;
    int64_t start = tokens_before + block_before(tokens, lds, &total), off = pages_before + block_before(pages, lds, &sum);
    /* (everybody has read the count) */
#pragma unroll
    for (int k = 0; k < PER; ++k) {
        const int64_t row = row0 + k;
        const int64_t end = start + (r[k].n > 0 ? r[k].n : 0), upto = off + r[k].pages;
        const bool good = r[k].good && end <= a.n_tokens;
        const bool served = good && (r[k].pages == 0 || upto <= have);
        if (row < a.n_rows) {
            const int32_t n = served ? r[k].n : 0;
            a.out_lengths[row] = n;
            a.starts[row] = start < a.n_tokens ? start : a.n_tokens;
            if (served) a.kv_lens[row] = r[k].old + n;
            if (a.status) a.status[row] = served ? 0u : good ? PARASON_KV_NO_PAGES : PARASON_KV_BAD_ROW;
            if (!FEW) a.off[row] = off;
            if (FEW) {
                first[tid] = (int32_t)(start < a.n_tokens ? start : a.n_tokens);
                olds[tid] = r[k].old, offs[tid] = (int32_t)(off < INT32_MAX ? off : INT32_MAX), taken[tid] = n;
            }
            /* The pages of the served rows: all before the first row that breaks a bound, which exactly one row is
             * (the sums only grow), or all there are. */
            const bool fits = upto <= have && end <= a.n_tokens;
            if (off <= have && start <= a.n_tokens && (!fits || row == a.n_rows - 1)) {
                const int64_t used = fits ? upto : off;
                *a.free_count = (int32_t)(have - used);
            }
            if (!FEW && one && row == 0) a.head[0] = have;
        }
        start = end, off = upto;
    }
    if (!FEW) return;
    __syncthreads();
    for (int32_t t = tid; t < a.n_tokens; t += TABLE_THREADS) {
        /* the last row that begins at or before t: empty rows in front of it begin there too */
        int32_t lo = 0, hi = (int32_t)a.n_rows;
        while (hi - lo > 1) {
            const int32_t mid = (lo + hi) >> 1;
            if (first[mid] <= t) lo = mid;
            else hi = mid;
        }
        const bool any = a.n_rows > 0;
        place_token(a, t, any && t - first[lo] < taken[lo], lo, t - first[lo], olds[lo], offs[lo], have);
    }
}

/* The last row of [lo, hi) that begins at or before t (row lo does); a wave's
 * lanes look at 64 rows at a time. */
__device__ __forceinline__ int64_t wave_row_of(const int64_t *starts, int64_t lo, int64_t hi, int64_t t)
{
    const int lane = (int)threadIdx.x & 63;
    while (hi - lo > 1) {
        const int64_t step = (hi - lo + 63) >> 6, i = lo + lane * step;
        const uint64_t there = __ballot(i < hi && starts[i < hi ? i : lo] <= t);
        const int64_t n = __builtin_popcountll(there);
        lo += (n - 1) * step;
        hi = lo + step < hi ? lo + step : hi;
    }
    return lo;
}

/* FILL_TOKENS tokens a block: the rows of its first and last one, the starts in
 * between in LDS, and then each token by itself. */
__global__ void __launch_bounds__(FILL_THREADS) table_fill(TableArgs a)
{
    __shared__ int64_t ends[2];
    __shared__ int32_t first[FILL_TOKENS], takes[FILL_TOKENS], olds[FILL_TOKENS], offs[FILL_TOKENS];
    const int64_t t0 = (int64_t)blockIdx.x * FILL_TOKENS;
    const int64_t t1 = t0 + FILL_TOKENS < a.n_tokens ? t0 + FILL_TOKENS : a.n_tokens; /* behind the last one */
    const int wave = (int)threadIdx.x >> 6;
    if (a.n_rows == 0) {
        for (int64_t t = t0 + threadIdx.x; t < t1; t += FILL_THREADS) place_token(a, t, false, 0, 0, 0, 0, 0);
        return;
    }
    if (wave < 2) {
        const int64_t row = wave_row_of(a.starts, 0, a.n_rows, wave ? t1 - 1 : t0);
        if ((threadIdx.x & 63) == 0) ends[wave] = row;
    }
    __syncthreads();
    const int64_t r0 = ends[0], n = ends[1] - r0 + 1;
    const bool held = n <= FILL_TOKENS; /* (more rows: most of them empty) */
    if (held)
        for (int i = (int)threadIdx.x; i < n; i += FILL_THREADS) {
            const int64_t d = a.starts[r0 + i] - t0, off = a.off[r0 + i];
            const int32_t n_taken = a.out_lengths[r0 + i];
            /* (the first row may begin before this block: -2^31 where that is further than 31 bits say, which a row that is
             * served never is) */
            first[i] = d < INT32_MIN ? INT32_MIN : (int32_t)d;
            takes[i] = n_taken, olds[i] = a.kv_lens[r0 + i] - n_taken, offs[i] = (int32_t)(off < INT32_MAX ? off : INT32_MAX);
        }
    __syncthreads();
    const int64_t have = a.head[0];
#pragma unroll
    for (int k = 0; k < FILL_PER; ++k) {
        const int32_t j = k * FILL_THREADS + (int32_t)threadIdx.x;
        const int64_t t = t0 + j;
        if (t >= t1) continue;
        if (held) {
            int32_t lo = 0, hi = (int32_t)n;
            while (hi - lo > 1) {
                const int32_t mid = (lo + hi) >> 1;
                if (first[mid] <= j) lo = mid;
                else hi = mid;
            }
            const int64_t in = (int64_t)j - first[lo];
            place_token(a, t, in < takes[lo], r0 + lo, in, olds[lo], offs[lo], have);
        } else {
            int64_t lo = 0, hi = n;
            while (hi - lo > 1) {
                const int64_t mid = (lo + hi) >> 1;
                if (a.starts[r0 + mid] <= t) lo = mid;
                else hi = mid;
            }
            const int64_t row = r0 + lo, in = t - a.starts[row];
            const int32_t taken = a.out_lengths[row];
            place_token(a, t, in < taken, row, in, a.kv_lens[row] - taken, a.off[row], have);
        }
    }
}

/* Page `nth` of a row goes onto the pool as the s-th of all that do. */
__device__ __forceinline__ void give_page(const TableArgs &a, int64_t row, int32_t nth, int64_t s, int64_t have, int64_t total)
{
    int32_t *const entry = a.pages + row * a.pages_stride + nth;
    const int64_t to = have + total - 1 - s;
    const int32_t page = *entry;
    *entry = -1;
    if (to < a.capacity) a.free_pages[to] = page;
    if ((page < 0 || to >= a.capacity) && a.status) atomicOr(&a.status[row], PARASON_KV_BAD_PAGE);
}

template <bool FEW>
__global__ void __launch_bounds__(TABLE_THREADS) table_shrink(TableArgs a)
{
    constexpr int PER = FEW ? 1 : TABLE_PER;
    __shared__ int64_t lds[TABLE_THREADS / 64];
    __shared__ int32_t offs[FEW ? FEW_ROWS : 1], keeps[FEW ? FEW_ROWS : 1];
    const int tid = (int)threadIdx.x;
    const int64_t row0 = (int64_t)blockIdx.x * TABLE_THREADS * PER + tid * PER;
    const bool one = gridDim.x == 1;
    int64_t before = 0, total = 0;
    if (!one) {
        int64_t p = 0, q = 0;
        for (int64_t i = tid; i < gridDim.x; i += TABLE_THREADS) {
            const int64_t s = a.tile_sums[2 * i + 1];
            p += i < blockIdx.x ? s : 0;
            q += s;
        }
        block_before(p, lds, &before);
        block_before(q, lds, &total);
    }
    const int64_t have = one ? free_pages_of(a) : a.head[0];
    TableRow r[PER];
    int64_t pages = 0, sum;
#pragma unroll
    for (int k = 0; k < PER; ++k) r[k] = table_row<false>(a, row0 + k), pages += r[k].pages;
    int64_t off = before + block_before(pages, lds, &sum);
    if (one) total = sum;
#pragma unroll
    for (int k = 0; k < PER; ++k) {
        const int64_t row = row0 + k;
        if (row < a.n_rows) {
            if (r[k].good) a.kv_lens[row] = r[k].n;
            else if (a.status) atomicOr(&a.status[row], PARASON_KV_BAD_ROW);
            if (FEW) offs[tid] = (int32_t)off, keeps[tid] = r[k].good ? pages_for(a, r[k].n) : 0;
            else a.off[row] = off;
            if (row == a.n_rows - 1) {
                if (!FEW) a.off[row + 1] = off + r[k].pages;
                const int64_t now = have + total;
                *a.free_count = (int32_t)(now < a.capacity ? now : a.capacity);
                if (!FEW && one) a.head[0] = have;
                if (!FEW) a.head[1] = total;
            }
        }
        off += r[k].pages;
    }
    if (!FEW) return;
    __syncthreads();
    for (int32_t s = tid; s < total; s += TABLE_THREADS) {
        int32_t lo = 0, hi = (int32_t)a.n_rows;
        while (hi - lo > 1) {
            const int32_t mid = (lo + hi) >> 1;
            if (offs[mid] <= s) lo = mid;
            else hi = mid;
        }
        give_page(a, lo, keeps[lo] + s - offs[lo], s, have, total);
    }
}

/* A wave takes up to GIVE_PAGES pages of a row. */
__global__ void __launch_bounds__(FILL_THREADS) table_give(TableArgs a, int64_t pieces)
{
    const int64_t unit = (int64_t)blockIdx.x * (FILL_THREADS / 64) + (threadIdx.x >> 6);
    const int64_t row = unit / pieces;
    if (row >= a.n_rows) return;
    const int64_t off = a.off[row];
    const int32_t n = (int32_t)(a.off[row + 1] - off), begin = (int32_t)(unit - row * pieces) * GIVE_PAGES;
    if (begin >= n) return;
    const int32_t end = begin + GIVE_PAGES < n ? begin + GIVE_PAGES : n, keeps = pages_for(a, a.kv_lens[row]);
    const int64_t have = a.head[0], total = a.head[1];
#pragma unroll 4
    for (int32_t i = begin + ((int32_t)threadIdx.x & 63); i < end; i += 64) give_page(a, row, keeps + i, off + i, have, total);
}

}  // namespace pk
