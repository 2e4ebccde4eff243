"""Scores far beyond what a softmax needs, of either sign: the position with the largest one is all that counts, and the
maximum that the weights are relative to must not be lost to its own rounding."""
import numpy as np
import pytest

from decoding_cases import Paged, torch_type
from gpu_util import log
from oracle import decoding_oracle as D
from paper_2608_24658_amd import parason as PX

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def dev():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    return torch.device("cuda:0")


@pytest.mark.parametrize("kind,given", [("bf16", "bf16"), ("fp16", "fp16"), ("fp8", "bf16"), ("int8", "fp16")])
@pytest.mark.parametrize("kv,length", [(200, 1), (200, 12), (250, 90), (5000, 1), (5000, 70)])
@pytest.mark.parametrize("scale", [2.0 ** 14, 2.0 ** 18, -2.0 ** 18, 2.0 ** 24, 2.0 ** 45])
def test_the_largest_score_takes_all(dev, kind, given, kv, length, scale):
    """Every position's score is a whole number of the scale, no two alike: e to the difference of any two is nothing."""
    log("case large scores %s as %s kv %d tokens %d scale %g" % (kind, given, kv, length, scale))
    rng = np.random.default_rng(kv + length)
    P = Paged(dev, [kv], 16, 1, 64, kind, seed=1)
    # values of 16 bits either way, and the codes keep them apart
    rank = rng.permutation(min(kv, 200))
    k, v = np.zeros((kv, 1, 64)), np.zeros((kv, 1, 64))
    k[:, 0, 0] = 1 + rank[np.arange(kv) % rank.size]
    if kv > rank.size:  # ties further on would share the weight: everything but the first ones far below
        k[rank.size:, 0, 1] = -1000.0 if scale > 0 else 1000.0
        k = np.concatenate([k[rank.size:], k[: rank.size]])
    v[:, 0] = rng.choice([-3.0, -2.0, -1.0, 1.0, 2.0, 3.0], (kv, 64))
    P.fill(lambda i, n: np.stack([k, v]))
    rows, total, starts = P.rows([length])
    q = torch.zeros(total, 4, 64)
    q[..., :2] = 1.0
    q[:, 1::2, 0] = -1.0  # (from the least on, too)
    out, lse = PX.tree_attention(q.to(dev).to(torch_type(given)), P.cache, rows, scale=scale, lse=True)
    out, lse = out.cpu().double().numpy(), lse.cpu().double().numpy()
    held_k, held_v = P.held[0]
    seen = D.visible(kv, length)
    for j in range(length):
        for h in range(4):
            s = (held_k[:, 0] @ q[j, h].double().numpy()) * scale
            s[~seen[j]] = -np.inf
            best = int(np.argmax(s))
            assert np.sum(s == s[best]) == 1
            want = held_v[best, 0]
            assert np.all(np.abs(out[j, h] - want) <= 2.0 ** -7 * np.abs(want)), (j, h, out[j, h][:4], want[:4])
            assert abs(lse[j, h] - s[best]) <= 2.0 ** -20 * abs(s[best]), (j, h, lse[j, h], s[best])
