"""Attention over a 4-bit cache whose scales make infinities (253 and 254, which a write does not make) where every token
of a block sees them: an infinite value is infinite in the results."""
import numpy as np
import pytest

from gpu_util import log
from oracle import serving_oracle as S
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
