/*
 * attn_kernels.h -- attention of a tree of tokens over the paged cache for
 * gfx950.
 *
 * A block takes the query heads that share a cache head, of neighbouring tokens
 * of one row, as the columns of its products, and runs over tiles of positions:
 *   S^T = K Q^T,   P^T = exp2(c S^T - max),   O^T += V^T P^T.
 * In S^T a lane of the 32x32 product holds 16 positions of one query, so the
 * maximum and the sum of a softmax are within the lane but for one exchange
 * with the lane 32 away, and P^T is already the right operand of the second
 * product: the 8 positions that a lane holds of each 16 are not consecutive
 * (0-3 and 8-11, or 4-7 and 12-15), which the rows of V^T are read to match.
 * V stays row by row in LDS; its transposed reads come from the LDS itself.
 *
 * Two shapes.  Few queries (blocks of 16 or 32 columns: single tokens, beams,
 * short drafts): the four waves take a quarter of each tile's positions each and
 * are joined at the end; what bounds it is reading the cache once.  128 single
 * tokens over 1.0 M positions of 8 heads of 128 FP8 values, 2.19 GB, take 436 us
 * (5.0 TB/s); 16 over 55,000 bfloat16 ones, 0.23 GB, 61 us (3.8 TB/s).
 * More queries: the waves take 32 columns each and share the tile; bound by the
 * products and the exponentials beside them.  A prompt of 8,192 tokens, 32
 * query heads over 8 of 128 values, 550 Gflop, takes 632 us (871 Tflop/s, where
 * a library product of 8192^3 reaches 1,348).  Long rows are cut into parts,
 * whose results tree_join puts together.  (Times of whole calls, among others.)
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
    int64_t q_stride_token, q_stride_head, out_stride_token, out_stride_head; /* elements */
    const uint64_t *mask;
    int64_t mask_stride;
    const int32_t *tree_lens;
    int32_t mask_words, n_q_heads, group;
    FastDiv group_div;
    float c2;            /* |scale| * log2(e), at least 2^-126 */
    bool negate;         /* scale < 0: the queries change their sign instead */
    bool q_wide, out_wide; /* queries in 16-byte, outputs in 8-byte pieces */
    int32_t q_blocks;    /* blocks of columns of a row and head */
    int32_t parts;       /* parts of a row's positions, part_len each (the last block of a row: the rest) */
    int32_t part_len;
    int64_t units;       /* rows * cache heads * parts */
    bool by_xcd;
    float *part_out;     /* [n_tokens * n_q_heads][parts][head_dim] */
    float2 *part_ml;     /* [n_tokens * n_q_heads][parts]: exponent of the maximum, sum */
};

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef short frag8 __attribute__((ext_vector_type(8)));
typedef short frag4 __attribute__((ext_vector_type(4)));
typedef float acc16 __attribute__((ext_vector_type(16)));
typedef float acc4 __attribute__((ext_vector_type(4)));
template <int CN>
struct Acc {
    typedef acc16 type;
};
template <>
struct Acc<16> {
    typedef acc4 type;
};

template <bool F16>
__device__ __forceinline__ acc4 mma(frag8 a, frag8 b, acc4 c)
{
    typedef __bf16 b8 __attribute__((ext_vector_type(8)));
    typedef _Float16 h8 __attribute__((ext_vector_type(8)));
    if (F16) return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(h8, a), __builtin_bit_cast(h8, b), c, 0, 0, 0);
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(b8, a), __builtin_bit_cast(b8, b), c, 0, 0, 0);
}

template <bool F16>
__device__ __forceinline__ acc16 mma(frag8 a, frag8 b, acc16 c)
{
    typedef __bf16 b8 __attribute__((ext_vector_type(8)));
    typedef _Float16 h8 __attribute__((ext_vector_type(8)));
    if (F16) return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(h8, a), __builtin_bit_cast(h8, b), c, 0, 0, 0);
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(b8, a), __builtin_bit_cast(b8, b), c, 0, 0, 0);
}

/* Two floats to two 16-bit values, rounded to nearest even. */
template <bool F16>
__device__ __forceinline__ uint32_t pack2(float x, float y)
{
    typedef __bf16 b2 __attribute__((ext_vector_type(2)));
    typedef _Float16 h2 __attribute__((ext_vector_type(2)));
    if (F16) return __builtin_bit_cast(uint32_t, h2{(_Float16)x, (_Float16)y});
    return __builtin_bit_cast(uint32_t, b2{(__bf16)x, (__bf16)y});
}

/* Four codes to four 16-bit values: exact in either type. */
template <bool F16, int KIND>
__device__ __forceinline__ uint2 widen4(uint32_t w)
{
    if (KIND == KV_FP8) {
        if (F16)
            return make_uint2(__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, 1.0f, false)),
                              __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, 1.0f, true)));
        return make_uint2(__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.0f, false)),
                          __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.0f, true)));
    }
    if (F16) {
        /* 1024 + (code + 128) is the float16 with the code in its low byte */
        typedef _Float16 h2 __attribute__((ext_vector_type(2)));
        const h2 off = {(_Float16)1152.0f, (_Float16)1152.0f};
        const uint32_t u = w ^ 0x80808080u;
        const h2 a = __builtin_bit_cast(h2, __builtin_amdgcn_perm(0x64646464u, u, 0x04010400u)) - off;
        const h2 b = __builtin_bit_cast(h2, __builtin_amdgcn_perm(0x64646464u, u, 0x04030402u)) - off;
        return make_uint2(__builtin_bit_cast(uint32_t, a), __builtin_bit_cast(uint32_t, b));
    }
    float x[4];
    int8x4_to_f32(w, x);
    return make_uint2(pack2<F16>(x[0], x[1]), pack2<F16>(x[2], x[3]));
}

/* Eight codes to the operand of a product. */
template <bool F16, int KIND>
__device__ __forceinline__ frag8 widen8(uint2 w)
{
    const uint2 a = widen4<F16, KIND>(w.x), b = widen4<F16, KIND>(w.y);
    return __builtin_bit_cast(frag8, make_uint4(a.x, a.y, b.x, b.y));
}

/* A word of V without its infinities and NaN, which become zeros. */
template <int KIND>
__device__ __forceinline__ uint32_t finite_word(uint32_t w)
{
    if (KIND == KV_INT8) return w;
    if (KIND == KV_FP8) {
        /* NaN is all ones below the sign: a zero byte of the complement */
        const uint32_t some = ((~w & 0x7F7F7F7Fu) + 0x7F7F7F7Fu) & 0x80808080u;
        return w & ((some >> 7) * 255u);
    }
    const uint32_t e = KIND == KV_F16 ? 0x7C00u : 0x7F80u;
    return w & (((w & e) != e ? 0x0000FFFFu : 0u) | (((w >> 16) & e) != e ? 0xFFFF0000u : 0u));
}

/* A value of the cache. */
template <int KIND>
__device__ __forceinline__ float cached_value(const char *p)
{
    if (KIND == KV_BF16) return bf16_to_f32(*reinterpret_cast<const uint16_t *>(p));
    if (KIND == KV_F16) return f16_to_f32(*reinterpret_cast<const uint16_t *>(p));
    float x[4];
    if (KIND == KV_FP8) fp8x4_to_f32((uint8_t)*p, x);
    else int8x4_to_f32((uint8_t)*p, x);
    return x[0];
}

constexpr int TREE_THREADS = 256;
constexpr int TREE_SKIP_WORDS = 64; /* of the list of a tree's tiles that nobody in the block sees: 2,048 tiles */

/* A block of COLS columns: 16 or 32 of them that all four waves take, or 128, 32 a wave. */
template <int DP, int COLS, int KIND>
struct TreeShape {
    static constexpr bool CODES = KIND == KV_FP8 || KIND == KV_INT8;
    /* Few columns: every wave has its own positions of a tile, and needs the others only at the end. */
    static constexpr bool SOLO = COLS < 128;
    /* Codes go to LDS as they are where one wave reads them again, and are widened behind it; where all four waves take
     * the same positions they are widened once, in front. */
    static constexpr bool RAW = CODES && SOLO;
    /* columns of a product, CN x CN results; the 64 / CN lanes of a column hold these positions of 32:
     * KSTEP * (i / 4) + 4 * (lane / CN) + i % 4, and these rows of O^T of CN: 8 * (i / 4) + 4 * (lane / CN) + i % 4 */
    static constexpr int CN = COLS == 16 ? 16 : 32, G = 64 / CN, NV = 32 / G, KSTEP = 128 / NV;
    static constexpr int AC = CN * CN / 64;           /* results a lane */
    static constexpr int WQ = COLS / CN;
    static constexpr int WK = 4 / WQ;                 /* waves that take the same columns */
    static constexpr int TK = SOLO ? 128 : 64;        /* positions of a tile */
    static constexpr int KW = TK / WK;                /* of it, those of one wave */
    static constexpr int SUBS = KW / 32;
    /* rows in LDS: 16 bytes more than a multiple of 128 spread the reads of K over the banks, 64 bytes more the
     * transposed reads of 16-bit V */
    static constexpr int ES = RAW ? 1 : 2;            /* bytes of a value in LDS */
    static constexpr int KS = RAW ? DP + 16 : DP + 8, VS = RAW ? DP + 16 : DP + 32; /* values */
    static constexpr int KBYTES = TK * KS * ES, VBYTES = TK * VS * ES;
    static constexpr int OS = DP + 4;                 /* floats of a row of the waves' results when they are joined */
    static constexpr int JOIN = (WK - 1) * COLS * OS * 4;
    /* blocks that a CU holds: by LDS, or by registers */
    static constexpr int BLOCKS = DP > 128 ? (COLS == 16 && RAW ? 2 : 1) : COLS > 16 ? (DP <= 64 && COLS == 32 ? 3 : 2) : RAW ? (DP <= 64 ? 4 : 3) : DP <= 64 ? 3 : 2;
    static constexpr int TILE = KBYTES + VBYTES > JOIN ? KBYTES + VBYTES : JOIN;
};

/* What a block's columns can see of their row, the same for the main kernel and the join. */
struct TreeSpan {
    int32_t tree, base;  /* tree positions, and the first of them */
    int32_t end;         /* positions that some column may see: [0, end) */
    int32_t tok0, tok1;  /* tokens of the columns: [tok0, tok1) */
    bool ok;
};

__device__ __forceinline__ TreeSpan tree_span(const TreeArgs &a, const KvRow &w, int64_t row, int32_t q_block, int cols)
{
    TreeSpan s;
    s.tree = a.mask ? (a.tree_lens ? a.tree_lens[row] : w.length) : 0;
    s.ok = w.ok && (!a.mask || (s.tree >= 0 && s.tree <= w.kv_len && ((int64_t)s.tree + 63) / 64 <= a.mask_words));
    s.base = w.kv_len - s.tree;
    const int64_t col0 = (int64_t)q_block * cols, n = (int64_t)w.length * a.group;
    const int64_t col1 = col0 + cols < n ? col0 + cols : n;
    s.tok0 = col0 < n ? (int32_t)div_by((uint32_t)col0, a.group_div) : w.length;
    s.tok1 = col0 < n ? (int32_t)div_by((uint32_t)(col1 - 1), a.group_div) + 1 : w.length;
    s.end = !s.ok ? 0 : a.mask ? w.kv_len : w.kv_len - w.length + s.tok1;
    if (s.end < 0) s.end = 0;
    return s;
}

__device__ __forceinline__ int32_t parts_of(const TreeArgs &a, int32_t end)
{
    const int32_t n = (int32_t)(((int64_t)end + a.part_len - 1) / a.part_len);
    return n < 1 ? 1 : n < a.parts ? n : a.parts;
}

template <int DP, int COLS, bool F16, int KIND>
__global__ void __launch_bounds__(TREE_THREADS, (TreeShape<DP, COLS, KIND>::BLOCKS)) tree_attention(TreeArgs a)
{
    typedef TreeShape<DP, COLS, KIND> Sh;
    constexpr int CN = Sh::CN, G = Sh::G, NV = Sh::NV, KSTEP = Sh::KSTEP, AC = Sh::AC, WQ = Sh::WQ;
    typedef typename Acc<CN>::type acc;
    constexpr int TK = Sh::TK, KS = Sh::KS, VS = Sh::VS, SUBS = Sh::SUBS;
    constexpr bool CODES = Sh::CODES, RAW = Sh::RAW;
    /* Type of the weights and of V: bfloat16 for codes, whose scales are in the weights.  The weights are rounded to it for
     * the matrix product: 2^-9 of each, against which a result of the same type is rounded by as much once more (bfloat16
     * results are off by 0.0020 to 0.0024 of their size in all, and by 0.0017 with float32 weights).  Two terms would take
     * half as many products again where products are what bounds the call. */
    constexpr bool PF16 = KIND == KV_F16;
    /* float16 results over codes: the weights go in as two bfloat16 terms, so that they are not the coarsest step of
     * the whole.  (float16 weights would lose all precision where the positions with nearly all of the weight hold a
     * code of zero.) */
    constexpr bool SPLIT = CODES && F16;
    /* The largest weight is 2^LIFT: of float16's 30 binades of full precision 29 are then below it. */
    constexpr int LIFT = PF16 ? 15 : 0;
    constexpr int VE = CODES ? 16 : 8;      /* values of a 16-byte piece of the cache */
    /* a tile's rows are loaded by the block, or its own ones by a wave */
    constexpr int LOADERS = Sh::SOLO ? 64 : TREE_THREADS, ROWS = Sh::SOLO ? Sh::KW : TK;
    constexpr int VPR = DP / VE, RPP = LOADERS / VPR, NP = ROWS / RPP;
    constexpr int ES = CODES ? 1 : 2;
    constexpr int KD = 8 * G, NK = DP / KD, ND = DP / CN;
    static_assert(NP >= 1 && NP * RPP == ROWS, "the loads cover a tile");

    __shared__ __attribute__((aligned(16))) char tile[Sh::TILE];
    __shared__ __attribute__((aligned(16))) float k_sc[CODES ? TK : 4], v_sc[CODES ? TK : 4];
    __shared__ int64_t place[TK];
    __shared__ int32_t v_stamp[TK];
    __shared__ uint32_t skip[TREE_SKIP_WORDS];
    __shared__ int32_t flags[2];            /* a bad page; the last tile with a value of V that is not finite (of the block) */
    __shared__ float join_ml[2][Sh::WK][COLS];
    char *const Ks = tile, *const Vs = tile + Sh::KBYTES;
    constexpr int LS = Sh::ES;              /* bytes of a value there */

    const int tid = (int)threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int n = lane % CN, h = lane / CN;
    const int wq = wave % WQ, wk = wave / WQ, k0 = wk * Sh::KW;

    /* ---- which row, cache head, part and columns */
    int64_t unit;
    int32_t q_block;
    if (a.by_xcd) {
        /* blocks that read the same keys on one XCD's L2 */
        const uint32_t x = blockIdx.x & 7u, y = blockIdx.x >> 3;
        unit = (int64_t)(y / (uint32_t)a.q_blocks) * 8 + x;
        q_block = (int32_t)(y % (uint32_t)a.q_blocks);
    } else {
        unit = blockIdx.x / (uint32_t)a.q_blocks;
        q_block = (int32_t)(blockIdx.x % (uint32_t)a.q_blocks);
    }
    if (unit >= a.units) return;
    q_block = a.q_blocks - 1 - q_block;     /* the longest of a chain first */
    const int32_t part = (int32_t)(unit % a.parts);
    const int32_t head = (int32_t)(unit / a.parts % a.c.n_heads);
    const int64_t row = unit / a.parts / a.c.n_heads;
    const KvRow w = load_row(a.r, a.c, row, false);
    const TreeSpan sp = tree_span(a, w, row, q_block, COLS);
    if (!sp.ok && part == 0 && head == 0 && q_block == 0 && tid == 0) report(a.r, row, PARASON_KV_BAD_ROW);
    if (!w.out_ok || sp.tok0 >= w.length) return;
    const int32_t my_parts = parts_of(a, sp.end);
    if (part >= my_parts) return;
    const int32_t k_begin = part * a.part_len;
    /* (a pool without pages: nothing is read, and what needs a position is NaN) */
    const int32_t k_end = a.c.n_pages == 0 ? k_begin : part == my_parts - 1 ? sp.end : k_begin + a.part_len;

    /* ---- this lane's query */
    const int32_t col = q_block * COLS + wq * CN + n;
    const int32_t tok = (int32_t)div_by((uint32_t)col, a.group_div);
    const bool live = tok < w.length;
    const int32_t q_head = head * a.group + (col - tok * a.group);
    const int64_t t = w.start + (live ? tok : 0);
    frag8 qf[NK];
    {
        const uint16_t *q = reinterpret_cast<const uint16_t *>(a.q) + t * a.q_stride_token + (live ? q_head : 0) * a.q_stride_head;
#pragma unroll
        for (int k = 0; k < NK; ++k) {
            const int d = k * KD + h * 8;
            uint4 x = make_uint4(0u, 0u, 0u, 0u);
            if (live && d < a.c.head_dim) {
                if (a.q_wide) {
                    x = *reinterpret_cast<const uint4 *>(q + d);
                } else {
                    uint32_t e[8];
                    for (int i = 0; i < 8; ++i) e[i] = q[d + i];
                    x = make_uint4(e[0] | (e[1] << 16), e[2] | (e[3] << 16), e[4] | (e[5] << 16), e[6] | (e[7] << 16));
                }
                if (a.negate) x.x ^= 0x80008000u, x.y ^= 0x80008000u, x.z ^= 0x80008000u, x.w ^= 0x80008000u;
            }
            qf[k] = __builtin_bit_cast(frag8, x);
        }
    }
    /* positions below `open` are seen by every column of the block */
    const int32_t open = a.mask ? sp.base : w.kv_len - w.length + sp.tok0 + 1;
    /* and this lane's own bound in a chain */
    const int32_t my_end = a.mask ? w.kv_len : (live ? w.kv_len - w.length + tok + 1 : 0);
    const uint64_t *const my_mask = a.mask ? a.mask + t * a.mask_stride : nullptr;
    const int32_t tree_words = (sp.tree + 63) >> 6;

    if (tid < 2) flags[tid] = tid == 0 && a.c.n_pages == 0 && sp.end > 0 ? 0 : -1;
    if (tid < TREE_SKIP_WORDS) skip[tid] = 0u;
    for (int i = tid; i < TK; i += TREE_THREADS) v_stamp[i] = -1;
    if (a.c.head_dim < DP)                   /* what is never loaded is zero */
        for (int i = tid * 16; i < Sh::KBYTES + Sh::VBYTES; i += TREE_THREADS * 16)
            *reinterpret_cast<uint4 *>(tile + i) = make_uint4(0u, 0u, 0u, 0u);
    __syncthreads();

    /* ---- the tree's tiles that some column sees: bit (tile - first tile of the tree) of `skip` */
    const int32_t tile0 = sp.base / TK;
    if (a.mask && sp.ok && k_end > sp.base) {   /* (a bad row's tree may be longer than its mask words) */
        const int32_t lo = k_begin > sp.base ? (k_begin - sp.base) >> 6 : 0;
        const int32_t words = ((k_end - sp.base + 63) >> 6) - lo;
        const int64_t total = (int64_t)words * (sp.tok1 - sp.tok0);
        if (total > (1 << 24)) {             /* (a list of 2,048 tiles would help such a tree little) */
            if (tid < TREE_SKIP_WORDS) skip[tid] = 0xFFFFFFFFu;
        } else for (uint32_t i = (uint32_t)tid; i < (uint32_t)total; i += TREE_THREADS) {
            const uint32_t j = i / (uint32_t)words;
            const int32_t x = lo + (int32_t)(i - j * (uint32_t)words);
            uint64_t m = a.mask[(w.start + sp.tok0 + j) * a.mask_stride + x];
            const int32_t rest = sp.tree - x * 64;
            if (rest < 64) m &= ~0ull >> (64 - rest);
            if (m == 0) continue;
            const int32_t p = sp.base + x * 64;
            const uint32_t first = (uint32_t)((p + __builtin_ctzll(m)) / TK - tile0);
            const uint32_t last = (uint32_t)((p + 63 - __builtin_clzll(m)) / TK - tile0);
            if (first < TREE_SKIP_WORDS * 32) atomicOr(&skip[first >> 5], 1u << (first & 31));
            if (last < TREE_SKIP_WORDS * 32) atomicOr(&skip[last >> 5], 1u << (last & 31));
        }
        __syncthreads();
    }
    const int32_t t_end = (k_end + TK - 1) / TK;
    auto next_tile = [&](int32_t x) {
        if (!a.mask) return x;
        while (x < t_end) {
            const uint32_t at = (uint32_t)(x - tile0);
            /* tiles with some of the prefix, and those behind the list, count as seen */
            if (x * TK < sp.base || at >= TREE_SKIP_WORDS * 32 || ((skip[at >> 5] >> (at & 31)) & 1u)) break;
            ++x;
        }
        return x;
    };

    /* ---- loads: a position's page a tile ahead of its keys and values, these a tile ahead of their use */
    const int32_t loader = Sh::SOLO ? lane : tid, row0 = Sh::SOLO ? k0 : 0; /* who loads what of a tile */
    const int32_t my_piece = loader % VPR, my_row = row0 + loader / VPR;
    const bool piece_live = my_piece * VE < a.c.head_dim;
    const int64_t piece_at = (int64_t)head * a.c.stride_head + (piece_live ? my_piece * VE : 0);
    const char *const kb = a.c.k + piece_at * ES, *const vb = a.c.v + piece_at * ES;
    auto together = [&]() {                  /* what a loader put into LDS is there for the others */
        if (!Sh::SOLO) {
            __syncthreads();
        } else {
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            __builtin_amdgcn_wave_barrier();
        }
    };
    /* Positions behind the part's last one read that again, and bad pages the pool's first value: every load has an
     * address, and what comes of these is masked, or NaN in the end. */
    int32_t pg = 0, pg_slot = 0;             /* of position row0 + loader of a tile */
    auto load_page = [&](int32_t x) {
        if (loader >= ROWS) return;
        const int32_t p = x * TK + row0 + loader;
        const uint32_t at = (uint32_t)(p < k_end ? p : k_end - 1), nth = div_by(at, a.c.page_div);
        pg_slot = (int32_t)(at - nth * (uint32_t)a.c.page_size);
        pg = a.r.pages[row * a.r.pages_stride + nth];
    };
    int64_t scale_at = 0;
    auto put_place = [&]() {
        if (loader >= ROWS) return;
        if (pg < 0 || pg >= a.c.n_pages) flags[0] = 0, pg = pg_slot = 0;
        place[row0 + loader] = (int64_t)pg * a.c.stride_page + (int64_t)pg_slot * a.c.stride_slot;
        if (CODES)
            scale_at = (int64_t)pg * a.c.scale_stride_page + (int64_t)pg_slot * a.c.scale_stride_slot +
                       (int64_t)head * a.c.scale_stride_head;
    };
    u32x4 kr[NP], vr[NP];
    float k_scale = 0.0f, v_scale = 0.0f;    /* of position row0 + loader */
    auto load_tile = [&]() {
#pragma unroll
        for (int p = 0; p < NP; ++p) {
            const int64_t from = place[my_row + p * RPP];
            kr[p] = *reinterpret_cast<const u32x4 *>(kb + from * ES);
            vr[p] = *reinterpret_cast<const u32x4 *>(vb + from * ES);
        }
        if (CODES && loader < ROWS) k_scale = a.c.k_scale[scale_at], v_scale = a.c.v_scale[scale_at];
    };
    uint64_t m_lo = 0, m_hi = 0;             /* mask words of a tile's positions of this wave */
    auto load_mask = [&](int32_t x) {
        const int32_t b = x * TK + k0 - sp.base;
        m_lo = m_hi = 0;
        if (a.mask && live && b + Sh::KW > 0) {
            const int32_t i = b < 0 ? 0 : b >> 6;
            if (i < tree_words) m_lo = my_mask[i];
            if (b >= 0 && i + 1 < tree_words) m_hi = my_mask[i + 1];
        }
    };

    acc o[ND] = {};
    float at = -INFINITY, l = 0.0f;          /* the exponent that o and l are relative to; this lane's share of the sum */

    /* tiles in turn: the one in work, and the one behind it */
    int32_t x = next_tile(k_begin / TK);
    int32_t x1 = x < t_end ? next_tile(x + 1) : t_end;
    if (x < t_end) {
        load_page(x);
        put_place();
        together();
        load_page(x1);
        load_mask(x);
        load_tile();
        together();
    }
    while (x < t_end) {
        const int32_t kp = x * TK;
        /* some column does not see all of the tile (of the wave's part of it) */
        const bool masked = kp + row0 + ROWS > open || kp + row0 + ROWS > k_end;
        /* ---- the tile goes to LDS; the next page's places (nobody reads the last ones any more) */
        put_place();
        if (CODES && loader < ROWS) k_sc[row0 + loader] = k_scale, v_sc[row0 + loader] = v_scale;
        bool odd_seen = false;
        if (masked && KIND != KV_INT8) {
            /* infinities and NaN of V reach only the queries that see them, for which a product by zero would not do:
             * they are left out here and added one position at a time below */
#pragma unroll
            for (int p = 0; p < NP; ++p) {
                const u32x4 v = vr[p];
                const u32x4 f = {finite_word<KIND>(v.x), finite_word<KIND>(v.y), finite_word<KIND>(v.z), finite_word<KIND>(v.w)};
                if (piece_live && ((f.x ^ v.x) | (f.y ^ v.y) | (f.z ^ v.z) | (f.w ^ v.w)) != 0u) {
                    v_stamp[my_row + p * RPP] = x;
                    odd_seen = true;
                }
                vr[p] = f;
            }
        }
        if (piece_live) {
#pragma unroll
            for (int p = 0; p < NP; ++p) {
                const int r = my_row + p * RPP;
                char *const kd = Ks + (r * KS + my_piece * VE) * LS, *const vd = Vs + (r * VS + my_piece * VE) * LS;
                if (CODES && !RAW) {
                    *reinterpret_cast<frag8 *>(kd) = widen8<F16, KIND>(make_uint2(kr[p].x, kr[p].y));
                    *reinterpret_cast<frag8 *>(kd + 16) = widen8<F16, KIND>(make_uint2(kr[p].z, kr[p].w));
                    *reinterpret_cast<frag8 *>(vd) = widen8<PF16, KIND>(make_uint2(vr[p].x, vr[p].y));
                    *reinterpret_cast<frag8 *>(vd + 16) = widen8<PF16, KIND>(make_uint2(vr[p].z, vr[p].w));
                    __builtin_amdgcn_sched_barrier(0);
                } else {
                    *reinterpret_cast<u32x4 *>(kd) = kr[p];
                    *reinterpret_cast<u32x4 *>(vd) = vr[p];
                }
            }
        }
        bool odd_values = false;             /* of the wave's positions, or of the block's */
        if (masked && KIND != KV_INT8) {
            if (Sh::SOLO) odd_values = __ballot(odd_seen) != 0;
            else if (odd_seen) flags[1] = x;
        }
        const uint64_t lo = m_lo, hi = m_hi;
        together();
        if (masked && KIND != KV_INT8 && !Sh::SOLO) odd_values = flags[1] == x;
        /* ---- the next one is on its way (loads come back in order, so what is needed first goes first) */
        const int32_t x2 = x1 < t_end ? next_tile(x1 + 1) : t_end;
        load_page(x2);
        load_mask(x1);
        load_tile();
        /* ---- S^T */
        float s[SUBS][NV];
        __builtin_amdgcn_s_setprio(1);       /* a wave in its products goes before one in its exponentials */
        /* the keys of a product are read KG products ahead */
        constexpr int KROWS = SUBS * (32 / CN), KG = NK < 4 ? NK : 4, KSTEPS = KROWS * NK / KG;
        auto read_keys = [&](int g, u32x4 *kf) {
            const char *ka = Ks + ((k0 + g * KG / NK * CN + n) * KS + h * 8) * LS;
#pragma unroll
            for (int j = 0; j < KG; ++j) {
                const int k = (g * KG + j) % NK;
                if (RAW) {
                    const uint2 c = *reinterpret_cast<const uint2 *>(ka + k * KD);
                    kf[j].x = c.x, kf[j].y = c.y;
                } else {
                    kf[j] = *reinterpret_cast<const u32x4 *>(ka + k * KD * 2);
                }
            }
        };
        u32x4 kf[KSTEPS + 1][KG];
        read_keys(0, kf[0]);
        acc c[KROWS];
#pragma unroll
        for (int i = 0; i < KROWS; ++i) c[i] = acc{};
#pragma unroll
        for (int g = 0; g < KSTEPS; ++g) {
            if (g + 1 < KSTEPS) read_keys(g + 1, kf[g + 1]);
#pragma unroll
            for (int j = 0; j < KG; ++j) {
                const frag8 f = RAW ? widen8<F16, KIND>(make_uint2(kf[g][j].x, kf[g][j].y)) : __builtin_bit_cast(frag8, kf[g][j]);
                c[g * KG / NK] = mma<F16>(f, qf[(g * KG + j) % NK], c[g * KG / NK]);
            }
            __builtin_amdgcn_sched_barrier(0);
        }
#pragma unroll
        for (int u = 0; u < SUBS; ++u) {
#pragma unroll
            for (int i = 0; i < 32 / CN; ++i)
#pragma unroll
                for (int r = 0; r < AC; ++r) s[u][i * AC + r] = c[u * (32 / CN) + i][r];
            if (CODES) {
#pragma unroll
                for (int i = 0; i < NV / 4; ++i) {
                    const float4 f = *reinterpret_cast<const float4 *>(&k_sc[k0 + u * 32 + KSTEP * i + 4 * h]);
                    s[u][4 * i] *= f.x, s[u][4 * i + 1] *= f.y, s[u][4 * i + 2] *= f.z, s[u][4 * i + 3] *= f.w;
                }
            }
        }
        __builtin_amdgcn_s_setprio(0);
        /* ---- what this lane's query sees of the wave's positions, from bit 0 on */
        uint32_t see[SUBS];
#pragma unroll
        for (int u = 0; u < SUBS; ++u) see[u] = 0xFFFFFFFFu;
        if (masked) {
#pragma unroll
            for (int u = 0; u < SUBS; ++u) {
                const int32_t p0 = kp + k0 + u * 32;
                const int32_t left = (my_end < k_end ? my_end : k_end) - p0;
                uint32_t m = left >= 32 ? 0xFFFFFFFFu : left <= 0 ? 0u : (1u << left) - 1u;
                if (a.mask) {
                    const int32_t b = p0 - sp.base;         /* of the wave's first word: u * 32 less */
                    const int32_t b0 = b - u * 32;
                    uint32_t tm;
                    if (b <= -32) {
                        tm = 0xFFFFFFFFu;
                    } else if (b < 0) {
                        tm = ((uint32_t)lo << -b) | ((1u << -b) - 1u);
                    } else {
                        /* lo holds word b0 / 64 (word 0 where the wave's positions begin in the prefix) */
                        const int32_t sh = b0 < 0 ? b : (b0 & 63) + u * 32;
                        tm = sh < 64 ? (uint32_t)(lo >> sh) | (sh > 32 ? (uint32_t)(hi << (64 - sh)) : 0u)
                                     : (uint32_t)(hi >> (sh - 64));
                    }
                    m &= tm;
                }
                see[u] = m;
                const uint32_t mine = m >> (4 * h);
#pragma unroll
                for (int r = 0; r < NV; ++r)
                    if (!((mine >> (KSTEP * (r / 4) + (r & 3))) & 1u)) s[u][r] = -INFINITY;
            }
        }
        /* ---- maximum, weights, sum */
        float top = s[0][0];
#pragma unroll
        for (int u = 0; u < SUBS; ++u)
#pragma unroll
            for (int r = 0; r < NV; ++r) top = fmaxf(top, s[u][r]);
#pragma unroll
        for (int k = CN; k < 64; k <<= 1) top = fmaxf(top, __shfl_xor(top, k));
        /* Exponents beyond FAR are rounded by more than a weight bears (the largest would be 2^(LIFT + 1) or, further on,
         * infinite or nothing): they are rounded down, and the weights that this takes over 2^LIFT are 2^LIFT, which
         * makes equal what the scores' own rounding does not tell apart for certain. */
        constexpr float FAR = 0x1p22f;
        float want = top * a.c2 - LIFT;
        want -= fabsf(want) >= FAR ? fminf(fabsf(want), 0x1p127f) * 0x1p-23f : 0.0f;
        const float at_new = fmaxf(at, want);
        const float ref = at_new == -INFINITY ? 0.0f : at_new;
        if (__ballot(at_new > at)) {
            const float corr = __builtin_amdgcn_exp2f(at - ref);
            l *= corr;
#pragma unroll
            for (int d = 0; d < ND; ++d)
#pragma unroll
                for (int r = 0; r < AC; ++r) o[d][r] *= corr;
            at = at_new;
        }
#pragma unroll
        for (int u = 0; u < SUBS; ++u)
#pragma unroll
            for (int r = 0; r < NV; ++r) s[u][r] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[u][r], a.c2, -ref));
        if (__ballot(fabsf(ref) >= FAR * (1.0f - 0x1p-20f))) {
            const float most = fabsf(ref) >= FAR * (1.0f - 0x1p-20f) ? (float)(1 << LIFT) : INFINITY;
#pragma unroll
            for (int u = 0; u < SUBS; ++u)
#pragma unroll
                for (int r = 0; r < NV; ++r) s[u][r] = s[u][r] > most ? most : s[u][r]; /* (NaN stays) */
        }
        float l4[4] = {};
#pragma unroll
        for (int u = 0; u < SUBS; ++u)
#pragma unroll
            for (int r = 0; r < NV; ++r) l4[r & 3] += s[u][r];
        l += (l4[0] + l4[1]) + (l4[2] + l4[3]);
        if (CODES) {
#pragma unroll
            for (int u = 0; u < SUBS; ++u) {
#pragma unroll
                for (int i = 0; i < NV / 4; ++i) {
                    const float4 f = *reinterpret_cast<const float4 *>(&v_sc[k0 + u * 32 + KSTEP * i + 4 * h]);
                    s[u][4 * i] *= f.x, s[u][4 * i + 1] *= f.y, s[u][4 * i + 2] *= f.z, s[u][4 * i + 3] *= f.w;
                }
                if (masked) {                /* no scale, whatever it is, makes a weight where nothing is seen */
                    uint32_t mine = see[u] >> (4 * h);
                    asm volatile("" : "+v"(mine)); /* (not worked out for the tiles that all see) */
#pragma unroll
                    for (int r = 0; r < NV; ++r)
                        if (!((mine >> (KSTEP * (r / 4) + (r & 3))) & 1u)) s[u][r] = 0.0f;
                }
            }
        }
        /* ---- O^T */
        __builtin_amdgcn_s_setprio(1);
        /* transposed reads: each 16 lanes name four (codes: eight) rows of 16 values and get a column each */
        const int g16 = CN == 32 ? ((lane >> 4) & 1) * 16 : 0, i16 = lane & 15;
        const char *va = RAW ? Vs + (k0 + 4 * h + ((i16 >> 1) & 3) + KSTEP * (i16 >> 3)) * VS + g16 + (i16 & 1) * 8
                             : Vs + ((k0 + 4 * h + (i16 >> 2)) * VS + g16 + (i16 & 3) * 4) * 2;
        constexpr int STEPS = SUBS * (NV / 8); /* products' worth of positions */
        auto read_values = [&](int g, u32x4 *vf) {
            typedef int int2v __attribute__((ext_vector_type(2)));
            typedef __attribute__((address_space(3))) frag4 lds4;
            typedef __attribute__((address_space(3))) int2v lds8;
#pragma unroll
            for (int d = 0; d < ND; ++d) {
                const char *v0 = va + ((g / (NV / 8) * 32 + g % (NV / 8) * 16) * VS + d * CN) * LS;
                if (RAW) {
                    const int2v f = __builtin_amdgcn_ds_read_tr8_b64_v2i32((lds8 *)v0);
                    vf[d].x = (uint32_t)f.x, vf[d].y = (uint32_t)f.y;
                } else {
                    const frag4 f0 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4 *)v0);
                    const frag4 f1 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4 *)(v0 + KSTEP * VS * LS));
                    vf[d] = __builtin_bit_cast(u32x4, (frag8)__builtin_shufflevector(f0, f1, 0, 1, 2, 3, 4, 5, 6, 7));
                }
            }
        };
        u32x4 vf[STEPS + 1][ND];             /* (codes: the first half) */
        read_values(0, vf[0]);
#pragma unroll
        for (int g = 0; g < STEPS; ++g) {
            const int u = g / (NV / 8), k = g % (NV / 8);
            if (g + 1 < STEPS) read_values(g + 1, vf[g + 1]);
            uint32_t pw[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) pw[i] = pack2<PF16>(s[u][8 * k + 2 * i], s[u][8 * k + 2 * i + 1]);
            const frag8 pf = __builtin_bit_cast(frag8, make_uint4(pw[0], pw[1], pw[2], pw[3]));
            frag8 pf_rest = {};
            if (SPLIT) {
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    pw[i] = pack2<PF16>(s[u][8 * k + 2 * i] - __uint_as_float(pw[i] << 16),
                                        s[u][8 * k + 2 * i + 1] - __uint_as_float(pw[i] & 0xFFFF0000u));
                pf_rest = __builtin_bit_cast(frag8, make_uint4(pw[0], pw[1], pw[2], pw[3]));
            }
#pragma unroll
            for (int d = 0; d < ND; ++d) {
                const frag8 v = RAW ? widen8<PF16, KIND>(make_uint2(vf[g][d].x, vf[g][d].y)) : __builtin_bit_cast(frag8, vf[g][d]);
                o[d] = mma<PF16>(v, pf, o[d]);
                if (SPLIT) o[d] = mma<PF16>(v, pf_rest, o[d]);
            }
            /* one step's values are read ahead, and no more: registers */
            __builtin_amdgcn_sched_barrier(0);
        }
        __builtin_amdgcn_s_setprio(0);
        if (odd_values) {
#pragma unroll
            for (int u = 0; u < SUBS; ++u) {
                for (int kk = 0; kk < 32; ++kk) {
                    const int r = k0 + u * 32 + kk;
                    if (v_stamp[r] != x) continue;
                    float p = 0.0f;
#pragma unroll
                    for (int i = 0; i < NV; ++i) p = (kk / KSTEP * 4 + (kk & 3)) == i ? s[u][i] : p;
                    p = __shfl(p, n + CN * (kk % KSTEP / 4));
                    if (!((see[u] >> kk) & 1u)) continue;
                    int32_t slot;
                    const int32_t page = page_of(a.r, a.c, row, kp + r < k_end ? kp + r : k_end - 1, &slot);
                    if (page < 0) continue;
                    int32_t h4 = 4 * h;      /* not known before: what depends on it is not worth registers in the loop */
                    asm volatile("" : "+v"(h4));
                    const char *v = a.c.v + ((int64_t)page * a.c.stride_page + (int64_t)slot * a.c.stride_slot +
                                             (int64_t)head * a.c.stride_head) * ES;
#pragma unroll
                    for (int d = 0; d < ND; ++d) {
#pragma unroll
                        for (int i = 0; i < AC; ++i) {
                            const int at_d = d * CN + 8 * (i / 4) + h4 + (i & 3);
                            if (at_d >= a.c.head_dim) continue;
                            const float e = cached_value<KIND>(v + at_d * ES);
                            if (!(e > -INFINITY && e < INFINITY)) o[d][i] += p * e;
                        }
                        __builtin_amdgcn_sched_barrier(0);
                    }
                }
            }
        }
        together();
        x = x1, x1 = x2;
    }
    __syncthreads();
    const bool bad = !sp.ok || flags[0] == 0;
    if (flags[0] == 0 && tid == 0) report(a.r, row, PARASON_KV_BAD_PAGE);

    /* ---- results */
#pragma unroll
    for (int k = CN; k < 64; k <<= 1) l += __shfl_xor(l, k);
    const float nan = __uint_as_float(0x7FC00000u);
    if (Sh::WK > 1) {
        /* the waves of the same columns: the maximum and the sum over them, then their shares of O, which the first
         * adds to its own */
        float *const Os = reinterpret_cast<float *>(tile);
        const int c = wq * CN + n;
        if (h == 0) join_ml[0][wk][c] = at, join_ml[1][wk][c] = l;
        __syncthreads();
        float top = -INFINITY, sum = 0.0f;
#pragma unroll
        for (int i = 0; i < Sh::WK; ++i) top = fmaxf(top, join_ml[0][i][c]);
        const float ref = top == -INFINITY ? 0.0f : top;
#pragma unroll
        for (int i = 0; i < Sh::WK; ++i) sum += join_ml[1][i][c] * __builtin_amdgcn_exp2f(join_ml[0][i][c] - ref);
        const float f = __builtin_amdgcn_exp2f(at - ref);
#pragma unroll
        for (int d = 0; d < ND; ++d)
#pragma unroll
            for (int i = 0; i < AC / 4; ++i) {
                o[d][4 * i] *= f, o[d][4 * i + 1] *= f, o[d][4 * i + 2] *= f, o[d][4 * i + 3] *= f;
                if (wk > 0)
                    *reinterpret_cast<float4 *>(&Os[((wk - 1) * COLS + c) * Sh::OS + d * CN + 8 * i + 4 * h]) =
                        make_float4(o[d][4 * i], o[d][4 * i + 1], o[d][4 * i + 2], o[d][4 * i + 3]);
            }
        at = top, l = sum;
        __syncthreads();
        if (wk > 0) return;
#pragma unroll
        for (int k = 0; k < Sh::WK - 1; ++k)
#pragma unroll
            for (int d = 0; d < ND; ++d)
#pragma unroll
                for (int i = 0; i < AC / 4; ++i) {
                    const float4 z = *reinterpret_cast<const float4 *>(&Os[(k * COLS + c) * Sh::OS + d * CN + 8 * i + 4 * h]);
                    o[d][4 * i] += z.x, o[d][4 * i + 1] += z.y, o[d][4 * i + 2] += z.z, o[d][4 * i + 3] += z.w;
                }
    }
    if (!live) return;
    if (bad) l = nan;
    const int64_t un = t * a.n_q_heads + q_head;
    if (my_parts > 1) {
        float *dst = a.part_out + (un * a.parts + part) * a.c.head_dim;
#pragma unroll
        for (int d = 0; d < ND; ++d)
#pragma unroll
            for (int i = 0; i < AC / 4; ++i) {
                const int at = d * CN + 8 * i + 4 * h;
                if (at < a.c.head_dim)
                    *reinterpret_cast<float4 *>(dst + at) = make_float4(o[d][4 * i], o[d][4 * i + 1], o[d][4 * i + 2], o[d][4 * i + 3]);
            }
        if (h == 0) a.part_ml[un * a.parts + part] = make_float2(at, l);
        return;
    }
    const float inv = l == 0.0f ? 0.0f : 1.0f / l;
    uint16_t *const dst = reinterpret_cast<uint16_t *>(a.out) + t * a.out_stride_token + q_head * a.out_stride_head;
#pragma unroll
    for (int d = 0; d < ND; ++d)
#pragma unroll
        for (int i = 0; i < AC / 4; ++i) {
            const int at = d * CN + 8 * i + 4 * h;
            if (at >= a.c.head_dim) continue;
            const uint2 p = make_uint2(pack2<F16>(o[d][4 * i] * inv, o[d][4 * i + 1] * inv),
                                       pack2<F16>(o[d][4 * i + 2] * inv, o[d][4 * i + 3] * inv));
            if (a.out_wide) *reinterpret_cast<uint2 *>(dst + at) = p;
            else dst[at] = (uint16_t)p.x, dst[at + 1] = (uint16_t)(p.x >> 16), dst[at + 2] = (uint16_t)p.y, dst[at + 3] = (uint16_t)(p.y >> 16);
        }
    if (h == 0 && a.lse) a.lse[un] = l == 0.0f ? -INFINITY : (at + __builtin_amdgcn_logf(l)) * 0.6931471805599453f;
}

/* A wave per (token, query head) joins the parts of its row: the parts' maxima
 * give their factors, the sums and the vectors are added in an order that the
 * sizes fix.  Four values a lane, so several parts at once. */
template <bool F16>
__global__ void __launch_bounds__(TREE_THREADS) tree_join(TreeArgs a, int cols)
{
    const int lane = (int)threadIdx.x & 63;
    const int64_t per_row = (int64_t)a.r.max_length * a.n_q_heads;
    const int64_t i = (int64_t)blockIdx.x * (TREE_THREADS / 64) + (threadIdx.x >> 6);
    const int64_t row = i / per_row;
    if (row >= a.r.n_rows) return;
    const int32_t tok = (int32_t)((uint32_t)(i - row * per_row) / (uint32_t)a.n_q_heads);
    const int32_t q_head = (int32_t)(i - row * per_row - (int64_t)tok * a.n_q_heads);
    const KvRow w = load_row(a.r, a.c, row, false);
    if (!w.out_ok || tok >= w.length) return;
    const int32_t col = tok * a.group + q_head % a.group;
    const TreeSpan sp = tree_span(a, w, row, col / cols, cols);
    const int32_t parts = parts_of(a, sp.end);
    if (parts == 1) return;
    const int64_t un = (w.start + tok) * a.n_q_heads + q_head;
    const float2 *ml = a.part_ml + un * a.parts;
    float m = -INFINITY;
    for (int32_t p = lane; p < parts; p += 64) m = fmaxf(m, ml[p].x);
#pragma unroll
    for (int k = 32; k > 0; k >>= 1) m = fmaxf(m, __shfl_xor(m, k));
    const float ref = m == -INFINITY ? 0.0f : m;
    int lanes = 4; /* of a part */
    while (lanes * 4 < a.c.head_dim) lanes <<= 1;
    const int at_once = 64 / lanes, d = (lane & (lanes - 1)) * 4;
    const bool mine = d < a.c.head_dim;
    const float *src = a.part_out + un * a.parts * a.c.head_dim + (mine ? d : 0);
    float4 y = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    float sum = 0.0f;
    auto add = [&](const float2 &v, const float4 &z) {
        const float f = __builtin_amdgcn_exp2f(v.x - ref);
        sum += v.y * f;
        y.x += z.x * f, y.y += z.y * f, y.z += z.z * f, y.w += z.w * f;
    };
    int32_t p = lane / lanes;
    for (; p + 3 * at_once < parts; p += 4 * at_once) {
        float2 v[4];
        float4 z[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            v[k] = ml[p + k * at_once];
            z[k] = *reinterpret_cast<const float4 *>(src + (int64_t)(p + k * at_once) * a.c.head_dim);
        }
#pragma unroll
        for (int k = 0; k < 4; ++k) add(v[k], z[k]);
    }
    for (; p < parts; p += at_once) add(ml[p], *reinterpret_cast<const float4 *>(src + (int64_t)p * a.c.head_dim));
    for (int k = 32; k >= lanes; k >>= 1) {
        sum += __shfl_xor(sum, k);
        y.x += __shfl_xor(y.x, k), y.y += __shfl_xor(y.y, k), y.z += __shfl_xor(y.z, k), y.w += __shfl_xor(y.w, k);
    }
    if (lane >= lanes || !mine) return;
    const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;
    const uint2 r = make_uint2(pack2<F16>(y.x * inv, y.y * inv), pack2<F16>(y.z * inv, y.w * inv));
    uint16_t *dst = reinterpret_cast<uint16_t *>(a.out) + (w.start + tok) * a.out_stride_token + q_head * a.out_stride_head + d;
    if (a.out_wide) *reinterpret_cast<uint2 *>(dst) = r;
    else dst[0] = (uint16_t)r.x, dst[1] = (uint16_t)(r.x >> 16), dst[2] = (uint16_t)r.y, dst[3] = (uint16_t)(r.y >> 16);
    if (lane == 0 && a.lse) a.lse[un] = sum == 0.0f ? -INFINITY : (m + __builtin_amdgcn_logf(sum)) * 0.6931471805599453f;
}

}  // namespace pk
