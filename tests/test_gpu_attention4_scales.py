"""Attention over a 4-bit cache whose scales make infinities (253 and 254, which a write does not make) where every token
of a block sees them: an infinite value is infinite in the results, and an infinite key's score takes all of the weight or
none of it."""
import numpy as np
import pytest

from decoding_cases import torch_type
from gpu_util import log
from oracle import decoding_oracle as D
from oracle import serving_oracle as S
from paper_2608_24658_amd import parason as PX
from serving_cases import Paged4
from test_gpu_attention4 import in_4_bits, run_case  # noqa: F401
from test_gpu_tree_attention import dev  # noqa: F401

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
GIVEN = pytest.mark.parametrize("given", ["bf16", "fp16"])


def put(P, what, row, pos, head, piece, codes, byte):
    """32 codes and their scale in place of those of a position, in the cache and in what the oracle takes it to hold."""
    pg, slot = (int(x) for x in P.place(row, pos))
    (P.cache.k, P.cache.v)[what].view(torch.uint8)[pg, slot, head, 16 * piece: 16 * piece + 16] = torch.from_numpy(S.pack4(codes)).to(P.dev)
    (P.cache.k_scale, P.cache.v_scale)[what].view(torch.uint8)[pg, slot, head, piece] = byte
    P.held[row][what][pos, head, 32 * piece: 32 * piece + 32] = S.values4(codes, np.array([byte], np.uint8))


@GIVEN
@pytest.mark.parametrize("dim", [96, 128, 256])
@pytest.mark.parametrize("lengths", [[1, 1], [4, 9], [40, 60]])
def test_infinite_values_that_all_see(dev, dim, lengths, given):  # noqa: F811
    """Values of 32 that a scale of 253 or 254 makes infinite, and a scale of 255, at the first positions of rows that go on
    for hundreds: tiles that no token sees in part."""
    log("case 4 bits infinite values that all see, dim %d tokens %s %s" % (dim, lengths, given))
    rng = np.random.default_rng(3)

    def spoil(P, seens):
        for i in range(len(lengths)):
            for byte, pos, piece in ((253, 5, 0), (254, 70, 1), (255, 130, 2)):
                put(P, 1, i, pos, i % 2, piece, rng.integers(0, 16, 32).astype(np.uint8), byte)

    for shape in (None, "tree"):
        out, _ = run_case(dev, 16, 2, 4, dim, [500, 330], lengths, shape=shape, seed=13, given=given, spoil=spoil)
        assert torch.isinf(out).any() and torch.isnan(out).any()


@GIVEN
@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("lengths", [[1, 1], [4, 9], [40, 60]])
def test_infinite_keys(dev, dim, lengths, given):  # noqa: F811
    """A key with one infinity, whose score is infinite: -inf is no weight, and the token's result is that of its other
    positions; inf leaves nothing but NaN.  Queries of few bits (one term holds them) and of all."""
    log("case 4 bits infinite keys, dim %d tokens %s %s" % (dim, lengths, given))
    rng = np.random.default_rng(4)
    heads, group, kv = 2, 4, [400, 200]
    for bits in (2, 10):
        P = Paged4(dev, kv, 16, heads, dim, "fp4", seed=1)
        P.fill(lambda i, n: rng.standard_normal((2, n, heads, dim)))
        spoiled = [[(3, 5), (150, dim - 1), (n - 1, 17)] for n in kv]  # position and value
        for i, places in enumerate(spoiled):
            for j, (pos, d) in enumerate(places):
                codes = np.zeros(32, np.uint8)
                codes[d % 32] = (6, 14, 7)[j]  # 4, -4, 6
                put(P, 0, i, pos, 1, d // 32, codes, (254, 253, 254)[j])
        rows, total, starts = P.rows(lengths)
        q = rng.standard_normal((total, heads * group, dim))
        q = torch.as_tensor(np.where(bits == 2, np.sign(q) * rng.integers(1, 4, q.shape), q)).to(torch_type(given))
        for i, n in enumerate(lengths):  # one token in two scores -inf everywhere
            for j, (_, d) in enumerate(spoiled[i]):
                at = q[starts[i]: starts[i] + n: 2, group:, d]
                at[:] = at.abs() * (-1.0, 1.0, -1.0)[j]
        out, lse = PX.tree_attention(q.to(dev), P.cache, rows, lse=True)
        out, lse, qh = out.cpu().double().numpy(), lse.cpu().double().numpy(), q.double().numpy()
        found = set()
        for i, n in enumerate(lengths):
            k, v = P.held[i]
            for t in range(n):
                for h in range(heads * group):
                    at, seen = starts[i] + t, D.visible(kv[i], int(n))[t: t + 1].copy()
                    kh, vh = k[:, h // group: h // group + 1], v[:, h // group: h // group + 1]
                    with np.errstate(invalid="ignore", over="ignore"):
                        s = kh[:, 0] @ qh[at, h]
                    if (s[seen[0]] == np.inf).any():
                        assert np.isnan(out[at, h]).all() and np.isnan(lse[at, h]), (i, t, h)
                        found.add("inf")
                        continue
                    found.add("-inf" if (s == -np.inf).any() else "none")
                    seen[0] &= s != -np.inf
                    o, z, ot, zt = D.attention(qh[at: at + 1, h: h + 1], np.where(np.isfinite(kh), kh, 0.0), vh, seen, dim ** -0.5, 7,
                                               dict(bf16=7, fp16=10)[given])
                    assert np.all(np.abs(out[at, h] - o[0, 0]) <= ot[0, 0]) and abs(lse[at, h] - z[0, 0]) <= zt[0, 0], (bits, i, t, h)
        assert "-inf" in found and "none" in found and (lengths == [1, 1] or "inf" in found)
