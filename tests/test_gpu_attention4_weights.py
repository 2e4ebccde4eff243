"""How exact the weights of the positions are over a 4-bit cache, where its results show it: two positions with values of
1 and -1 and nearly the same weight, which all but cancel."""
import numpy as np
import pytest

from gpu_util import log
from paper_2608_24658_amd import parason as PX
from serving_cases import Paged4
from test_gpu_tree_attention import dev, torch_type  # noqa: F401

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("given", ["bf16", "fp16"])
@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("tokens,group", [(1, 4), (3, 16), (16, 4)])
def test_two_positions_that_all_but_cancel(dev, given, dim, tokens, group):  # noqa: F811
    """Scores of 0 and -d, d some 2^-10: the result is (1 - exp(-d)) / (1 + exp(-d)).  A weight of two bfloat16 terms is off
    by 2^-17 of itself and float32's exponential, sum and quotient by a few 2^-22, over a sum of nearly 2: 2^-17 in all, on
    top of the result's own rounding.  (With one term it would be up to 2^-10, half of d.)"""
    log("case 4 bits cancelling weights dim %d tokens %d group %d %s" % (dim, tokens, group, given))
    P = Paged4(dev, [tokens + 1], 16, 1, dim, "fp4", seed=0)

    def values(i, n):
        x = np.zeros((2, n, 1, dim))
        x[0, 1, 0, 0], x[1, 0], x[1, 1] = -1.0, 1.0, -1.0
        return x

    P.fill(values)
    rows, total, _ = P.rows([tokens])
    mask = torch.full((total, 1), 1, dtype=torch.int64, device=dev)  # the prefix and the tree's first position
    q = torch.zeros(total, group, dim)
    q[..., 0] = (torch.arange(total * group).view(total, group) % 31 + 1) / 1024
    got = PX.tree_attention(q.to(torch_type(given)).to(dev), P.cache, rows, mask=mask, scale=1.0).cpu().double().numpy()
    d = q[..., 0].double().numpy()[..., None]
    want = np.tanh(d / 2)
    assert np.all(np.abs(got - want) <= 2.0 ** -17 + want * {"bf16": 2.0 ** -8, "fp16": 2.0 ** -11}[given])
