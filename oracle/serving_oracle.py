"""The cache's tables, the norm and rotation of queries and keys, and 4-bit values, one after the other as the definitions
of ``include/parason.h`` say it (plain numpy, 64 bits)."""
import numpy as np

GRID4 = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
BAD_ROW, BAD_PAGE, NO_PAGES = 1, 2, 4
MAX_LEN = 1 << 30


# ---- 4-bit values ----------------------------------------------------------------------------------------------------


def quantise4(x):
    """(codes, scale bytes) of float32 heads [..., dim]: codes [..., dim] 0 .. 15, bytes [..., dim / 32]."""
    x = np.asarray(x, np.float32).astype(np.float64)
    g = x.reshape(x.shape[:-1] + (x.shape[-1] // 32, 32))
    fine = np.isfinite(g).all(-1)
    amax = np.where(fine, np.abs(np.where(np.isfinite(g), g, 0)).max(-1), 0.0)
    e = np.full(amax.shape, 125)
    for k in range(125, -121, -1):
        e = np.where(amax <= 7 * 2.0 ** k, k, e)
    y = np.where(fine[..., None], g, 0.0) / 2.0 ** e[..., None]
    a = np.abs(y)
    # the nearest value; of two that are as near the one with the even code
    hi = np.clip(np.searchsorted(GRID4, a), 1, 7)
    lo = hi - 1
    down, up = a - GRID4[lo], GRID4[hi] - a
    code = np.where(down < up, lo, np.where(up < down, hi, np.where(lo % 2 == 0, lo, hi)))
    code = code + np.where(np.signbit(y), 8, 0)
    return code.reshape(x.shape).astype(np.uint8), np.where(fine, e + 127, 255).astype(np.uint8)


def values4(codes, scales):
    """The float32 values that codes and scale bytes stand for: exact."""
    x = np.where(codes & 8, -1.0, 1.0) * GRID4[codes & 7]
    s = np.where(scales == 255, np.nan, 2.0 ** (scales.astype(np.float64) - 127))
    with np.errstate(over="ignore"):
        return (x.reshape(x.shape[:-1] + (x.shape[-1] // 32, 32)) * s[..., None]).reshape(x.shape).astype(np.float32)


def pack4(codes):
    """Two codes a byte, the first in the low half."""
    return (codes[..., 0::2] | codes[..., 1::2] << 4).astype(np.uint8)


def unpack4(packed):
    return np.stack([packed & 15, packed >> 4], -1).reshape(packed.shape[:-1] + (2 * packed.shape[-1],))


# ---- tables ----------------------------------------------------------------------------------------------------------


def extend(free, count, kv_lens, pages, lengths, page_size, n_tokens):
    """kv_extend on numpy arrays, in place; returns (count, dict)."""
    n, max_pages = pages.shape
    capacity = free.size
    have = min(max(int(count), 0), capacity)
    out = dict(lengths=np.zeros(n, np.int32), starts=np.zeros(n, np.int64), status=np.zeros(n, np.uint32),
               positions=np.full(n_tokens, -1, np.int32), slots=np.full(n_tokens, -1, np.int64), rows=np.full(n_tokens, -1, np.int32))
    most = min(max_pages * page_size, MAX_LEN)
    start = wanted = used = 0
    for i in range(n):
        wish, old = int(lengths[i]), int(kv_lens[i])
        out["starts"][i] = min(start, n_tokens)
        here, start = start, start + max(wish, 0)
        if wish < 0 or old < 0 or old + wish > most:
            out["status"][i] = BAD_ROW
            continue
        had, need = -(-old // page_size), -(-(old + wish) // page_size) - -(-old // page_size)
        wanted += need
        if start > n_tokens:
            out["status"][i] = BAD_ROW
            continue
        if need and wanted > have:
            out["status"][i] = NO_PAGES
            continue
        for k in range(need):
            used += 1
            pages[i, had + k] = free[have - used]
        for j in range(wish):
            p = old + j
            out["positions"][here + j], out["rows"][here + j] = p, i
            page = int(pages[i, p // page_size])
            out["slots"][here + j] = page * page_size + p % page_size if page >= 0 else -1
        out["lengths"][i] = wish
        kv_lens[i] = old + wish
    # (a count out of bounds counts as the nearer bound, which is what it becomes)
    return have - used, out


def shrink(free, count, kv_lens, pages, new_lens, page_size, status):
    """kv_shrink on numpy arrays, in place; returns the count."""
    n, max_pages = pages.shape
    have = min(max(int(count), 0), free.size)
    most = min(max_pages * page_size, MAX_LEN)
    gone = []
    for i in range(n):
        new, old = int(new_lens[i]), int(kv_lens[i])
        if new < 0 or new > old or old > most:
            status[i] |= BAD_ROW
            continue
        gone += [(i, k) for k in range(-(-new // page_size), -(-old // page_size))]
        kv_lens[i] = new
    for s, (i, k) in enumerate(gone):
        to = have + len(gone) - 1 - s
        if to < free.size:
            free[to] = pages[i, k]
        if to >= free.size or pages[i, k] < 0:
            status[i] |= BAD_PAGE
        pages[i, k] = -1
    return min(have + len(gone), free.size)


# ---- norm and rotation -----------------------------------------------------------------------------------------------


def _pairs(dim, turned, interleaved):
    j = np.arange(turned // 2)
    return (2 * j, 2 * j + 1) if interleaved else (j, j + turned // 2)


def rotate(x, weight, positions, freqs, eps, interleaved):
    """y and a bound of its error before it is rounded, for heads x [tokens, heads, dim] in 64 bits.

    In units u = 2^-24 (half an ulp, relative): the mean of the squares has at most 16 products summed in a lane, 4 sums
    over lanes, and the product with a rounded 1 / dim: 22 u, so its root 11 u, and 1 / root 2 u more; the products with
    x and the weight 2 u: 15 u.  A cosine or sine is off by 2 ulp (4 u) and its correction 2 u; each of the two terms of
    a rotated value has a product and a sum: 2 u more.  23 u of |n_a| + |n_b| in all; 32 u are allowed.  The angle is a
    product of doubles, off by 2^-52 of its size in all."""
    x = np.asarray(x, np.float64)
    dim = x.shape[-1]
    n = x / np.sqrt((x * x).mean(-1, keepdims=True) + eps) * (1.0 if weight is None else weight)
    y, size = n.copy(), np.abs(n)
    a, b = _pairs(dim, 2 * freqs.size, interleaved)
    angle = positions[:, None, None] * freqs
    c, s = np.cos(angle), np.sin(angle)
    y[..., a], y[..., b] = n[..., a] * c - n[..., b] * s, n[..., b] * c + n[..., a] * s
    size[..., a] = size[..., b] = np.abs(n[..., a]) + np.abs(n[..., b])
    far = np.zeros(size.shape)
    far[..., a] = far[..., b] = np.abs(angle) * 2.0 ** -51
    y[positions < 0], size[positions < 0] = 0.0, 0.0
    return y, size * (32 * 2.0 ** -24 + far)


def rotate_grad(x, dy, weight, positions, freqs, eps, interleaved):
    """dx, dw, and bounds of their errors (dx before it is rounded), in 64 bits.

    The gradient turned back is off by 8 u of |a| + |b| (as above), a normed value by 14 u; dx's two terms have some more
    products and a sum over dim terms: 64 u of their sizes are allowed.  dw adds one term for each token and head, in
    float32 in a lane and over lanes: at most as many roundings as there are terms, on top of 32 u for each term."""
    x, dy = np.asarray(x, np.float64), np.asarray(dy, np.float64)
    dim = x.shape[-1]
    there = (positions >= 0)[:, None, None]
    x, dy = np.where(there, x, 0.0), np.where(there, dy, 0.0)
    w = np.ones(dim) if weight is None else np.asarray(weight, np.float64)
    g, size = dy.copy(), np.abs(dy)
    a, b = _pairs(dim, 2 * freqs.size, interleaved)
    angle = positions[:, None, None] * freqs
    c, s = np.cos(angle), np.sin(angle)
    g[..., a], g[..., b] = dy[..., a] * c + dy[..., b] * s, dy[..., b] * c - dy[..., a] * s
    size[..., a] = size[..., b] = np.abs(dy[..., a]) + np.abs(dy[..., b])
    far = np.abs(np.where(there, angle, 0.0)).max(initial=0.0) * 2.0 ** -51
    r = 1 / np.sqrt((x * x).mean(-1, keepdims=True) + eps)
    h = x * r
    dw = (g * h).sum((0, 1))
    gw = g * w
    dx = r * (gw - h * (gw * h).mean(-1, keepdims=True))
    size_w = size * np.abs(w)
    dx_tol = r * (size_w + np.abs(h) * (size_w * np.abs(h)).mean(-1, keepdims=True)) * (64 * 2.0 ** -24 + far)
    dw_tol = (size * np.abs(h)).sum((0, 1)) * ((32 + x.shape[0] * x.shape[1]) * 2.0 ** -24 + far) + 2.0 ** -24 * np.abs(dw)
    return np.where(there, dx, 0.0), dw, np.where(there, dx_tol, 0.0), dw_tol
