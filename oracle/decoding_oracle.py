"""The paged cache, the attention of a tree of tokens over it, and the beams, in 64 bits (plain numpy).

The definitions are those of ``include/parason.h``.  Quantised values are exact: the scale is a float32
product with the rounded 1 / Q and the code a float32 quotient, rounded once.  The attention also gives, for every output, a bound of the error that float32 scores
and sums and 16-bit weights may have (see ``attention``).
"""
import numpy as np

E4M3 = np.array([(-1.0 if c & 128 else 1.0) * ((c & 7) / 8 * 2.0 ** -6 if (c >> 3) & 15 == 0 else
                 (1 + (c & 7) / 8) * 2.0 ** (((c >> 3) & 15) - 7)) if c & 127 != 127 else np.nan for c in range(256)])


def fp8_codes(x):
    """Codes of the e4m3 values nearest to x (|x| <= 448), ties to the even code."""
    grid = E4M3[:127]
    a = np.abs(x)
    hi = np.clip(np.searchsorted(grid, a), 1, 126)
    lo = hi - 1
    down, up = a - grid[lo], grid[hi] - a
    code = np.where(down < up, lo, np.where(up < down, hi, np.where(lo % 2 == 0, lo, hi)))
    return (code | np.where(np.signbit(x), 128, 0)).astype(np.uint8)


def quantise(x, kind):
    """(codes, scales) of float32 heads [..., dim]; kind "fp8" or "int8"."""
    x = np.asarray(x, dtype=np.float32)
    top = np.float32(448.0 if kind == "fp8" else 127.0)
    amax = np.abs(x).max(-1)
    with np.errstate(invalid="ignore", over="ignore"):
        scale = np.maximum(amax * (np.float32(1) / top), np.float32(2.0 ** -126)).astype(np.float32)
        fine = np.isfinite(x).all(-1)
        q = np.where(fine[..., None], x / np.where(fine, scale, 1)[..., None], np.float32(0)).astype(np.float32)
    codes = fp8_codes(q.astype(np.float64)) if kind == "fp8" else np.rint(q).astype(np.int8)
    return codes, np.where(fine, scale, np.float32(np.nan))


def values(codes, scales, kind):
    """float32 values that codes stand for: one product, rounded once."""
    x = E4M3[codes.view(np.uint8)].astype(np.float32) if kind == "fp8" else codes.view(np.int8).astype(np.float32)
    return x * scales[..., None]


def visible(kv_len, length, tree_len=None, mask=None):
    """[length, kv_len] truth values; mask: uint64 words [length, words] of the row's tokens."""
    p = np.arange(kv_len)
    if mask is None:
        return p[None, :] <= (kv_len - length + np.arange(length))[:, None]
    tree_len = length if tree_len is None else tree_len
    bit = p - (kv_len - tree_len)
    word = np.clip(bit // 64, 0, max(0, mask.shape[1] - 1))
    seen = np.ones((length, kv_len), bool)
    tree = bit >= 0
    if tree.any():
        seen[:, tree] = (mask[:, word[tree]] >> (bit[tree] % 64).astype(np.uint64)) & np.uint64(1) != 0
    return seen


def attention(q, k, v, seen, scale, weight_bits, out_bits):
    """One row: q [n, q_heads, dim], k and v [kv, heads, dim] (64-bit values of what the cache holds), seen [n, kv].

    Returns out, lse, and bounds of their errors: the scores are sums of `dim` products in float32 (2 dim + 16 roundings
    of half an ulp of the sum of magnitudes, a factor of two for sums in blocks), exp adds 2^-21, the sums over the
    positions one rounding each, a weight one rounding to `weight_bits` bits of fraction (float16: or to a multiple of
    2^-24, its smallest step) and the output one to `out_bits`.
    """
    n, q_heads, dim = q.shape
    kv, heads, _ = k.shape
    out, lse = np.zeros((n, q_heads, dim)), np.full((n, q_heads), -np.inf)
    out_tol, lse_tol = np.zeros((n, q_heads, dim)), np.zeros((n, q_heads))
    eps = 2.0 ** -24
    for h in range(q_heads):
        kh, vh = k[:, h // (q_heads // heads)], v[:, h // (q_heads // heads)]
        for i in range(n):
            at = np.nonzero(seen[i])[0]
            if at.size == 0:
                continue
            with np.errstate(invalid="ignore", over="ignore"):
                s = kh[at] @ q[i, h] * scale
                if np.all(s == -np.inf):
                    continue
                e = np.exp(s - s.max())
                p = e / e.sum()
                out[i, h] = p @ vh[at]
                lse[i, h] = s.max() + np.log(e.sum())
                size = (np.abs(kh[at]) @ np.abs(q[i, h])).max() * abs(scale)
                ds = (2 * dim + 16) * eps * size + 2.0 ** -21
                weights = p @ np.abs(vh[at])
                tiny = 2.0 ** -25 * np.abs(vh[at]).sum(0) / e.sum() if weight_bits == 10 else 0.0
                out_tol[i, h] = weights * (1.01 * 2.0 ** -(weight_bits + 1) + 2 * ds + 2 * at.size * eps) + tiny \
                    + np.abs(out[i, h]) * 2.0 ** -(out_bits + 1) + 2.0 ** (-25 if out_bits == 10 else -133)
                lse_tol[i, h] = ds + at.size * eps + 2 * eps * abs(lse[i, h])
    return out, lse, out_tol, lse_tol


def beam_candidates(logits, scores, flags, beams, done=2):
    """Scores [groups, beams * (vocab + 1)] in 64 bits: place (beam, token + 1), -inf: no candidate."""
    x = np.asarray(logits, dtype=np.float64)
    rows, vocab = x.shape
    out = np.full((rows, vocab + 1), -np.inf)
    for r in range(rows):
        if not np.isfinite(scores[r]):
            continue
        if flags[r]:
            if flags[r] == done:
                out[r, 0] = scores[r]
            continue
        top = x[r].max()
        if not np.isfinite(top) or np.isnan(x[r]).any():
            continue
        out[r, 1:] = scores[r] + (x[r] - (top + np.log(np.exp(x[r] - top).sum())))
    return out.reshape(rows // beams, beams * (vocab + 1))


def beam_select(candidates, beams):
    """Places of the best candidates of every group, best first, ties to the lowest; -1 where there are none left."""
    out = np.full((candidates.shape[0], beams), -1, np.int64)
    for g, c in enumerate(candidates):
        order = np.lexsort((np.arange(c.size), -c))[:beams]
        order = order[c[order] > -np.inf]
        out[g, : order.size] = order
    return out


def beam_lse(x):
    """ln sum exp of a row of logits in 64 bits, and as beam_select has it: the logarithm of sum exp(x - top) rounded to
    float32 (there: a unit in the last place at most), then its sum with top."""
    x = np.asarray(x, dtype=np.float64)
    top = x.max()
    ln = np.log(np.exp(x - top).sum())
    return top + ln, np.float32(top) + np.float32(ln)


def beam_scores(logits, scores, flags, beams, done=2, lse=None):
    """The float32 scores of beam_candidates' places as beam_select rounds them: score + (logit - lse), each step once.
    lse: the rows' own, where the last place of the logarithm matters."""
    x = np.asarray(logits, dtype=np.float32)
    scores = np.asarray(scores, dtype=np.float32)
    rows, vocab = x.shape
    out = np.full((rows, vocab + 1), -np.inf, np.float32)
    for r in range(rows):
        if not np.isfinite(scores[r]):
            continue
        if flags[r]:
            if flags[r] == done:
                out[r, 0] = scores[r]
            continue
        if not np.isfinite(x[r].max()) or np.isnan(x[r]).any():
            continue
        out[r, 1:] = scores[r] + (x[r] - (beam_lse(x[r])[1] if lse is None else np.float32(lse[r])))
    return out.reshape(rows // beams, beams * (vocab + 1))
