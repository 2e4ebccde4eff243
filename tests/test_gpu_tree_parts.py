"""What the bounds of the attention's other tests are too wide to see: a position lost or counted twice where a row is
cut into parts and tiles, and the second term of the weights where float16 results come from 8-bit caches."""
import numpy as np
import pytest

import test_gpu_tree_attention as T
from decoding_cases import Paged, torch_type, tree_seen, words
from gpu_util import log
from oracle import decoding_oracle as D
from paper_2608_24658_amd import parason as PX
from test_gpu_tree_attention import dev  # noqa: F401

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kind", ["bf16", "fp16", "fp8", "int8"])
@pytest.mark.parametrize("kv_lens,lengths,group,tree", [
    ([9000, 4001, 513, 63], [1, 1, 1, 1], 4, None),                  # blocks of 16 columns, the shortest parts
    ([9100, 2049, 31], [3, 4, 3], 8, None),                          # 32
    ([9100, 5000, 1, 4097], [150, 40, 1, 2], 2, None),               # 128, ragged
    ([33000], [1], 4, None),                                         # more parts than a wave joins at once
    ([4500, 130], [20, 20], 2, (3000, 130)),                         # a long tree of threads
    ([4500, 700], [90, 70], 2, (4400, 650)),
])
def test_every_position_counts_once(dev, kind, kv_lens, lengths, group, tree):  # noqa: F811
    """Keys of zero, so that every position seen has the same weight, and as values one one among zeros, in dimension
    (position % 256): result d times the number of positions seen is the number of those that belong to d, some tens.  One
    position more or less is a change of 1 / 130 or more; the weights are equal powers of two, so the error is the sum's
    (kv additions in float32, 2^-24 each), the scale's of a code (2^-9: its weight is rounded to bfloat16) and the
    result's rounding (2^-9 in bfloat16): 1 / 170 in all.  (The values of codes: 127 or 448 times the scale, exact.)"""
    log("case every position once %s kv %s tokens %s" % (kind, kv_lens, lengths))
    dim = 256
    given = "bf16" if kind == "bf16" else "fp16"
    P = Paged(dev, kv_lens, 24, 1, dim, kind, seed=2)

    def values(i, n):
        x = np.zeros((2, n, 1, dim))
        x[1, np.arange(n), 0, np.arange(n) % dim] = 1.0
        return x

    P.fill(values)
    rows, total, starts = P.rows(lengths)
    q = torch.as_tensor(np.random.default_rng(0).standard_normal((total, group, dim)).astype(np.float32)).to(torch_type(given))
    mask = trees = None
    seens = [D.visible(int(kv), int(n)) for kv, n in zip(kv_lens, lengths)]
    if tree:
        rng = np.random.default_rng(1)
        n_words = -(-max(tree) // 64)
        made = [words(tree_seen(rng, t, "threads")[t - n:], n_words) for t, n in zip(tree, lengths)]
        mask = torch.as_tensor(np.concatenate(made).view(np.int64)).to(dev)
        trees = torch.tensor(tree, dtype=torch.int32, device=dev)
        seens = [D.visible(int(kv), int(n), int(t), m) for kv, n, t, m in zip(kv_lens, lengths, tree, made)]
    out, lse = PX.tree_attention(q.to(dev), P.cache, rows, mask=mask, tree_lens=trees, lse=True)
    out, lse = out.cpu().double().numpy(), lse.cpu().double().numpy()
    for i, n in enumerate(lengths):
        for j in range(n):
            seen = np.nonzero(seens[i][j])[0]
            want = np.bincount(seen % dim, minlength=dim) * 1.0
            for h in range(group):
                got = out[starts[i] + j, h] * seen.size
                assert np.all(np.abs(got - want) <= want / 170), (i, j, h, got[:4], want[:4])
                assert abs(lse[starts[i] + j, h] - np.log(seen.size)) <= (seen.size + 16) * 2.0 ** -24 * max(1.0, np.log(seen.size))


@pytest.mark.parametrize("kind", ["fp8", "int8"])
@pytest.mark.parametrize("case", [
    dict(page=16, heads=2, group=4, dim=64, kv_lens=[1, 17, 64, 129, 700], lengths=[1] * 5),
    dict(page=16, heads=1, group=2, dim=128, kv_lens=[300, 2500], lengths=[20, 9]),
    dict(page=24, heads=1, group=5, dim=96, kv_lens=[210, 90], lengths=[150, 90]),
    dict(page=16, heads=2, group=3, dim=64, kv_lens=[8, 40, 267], lengths=[8, 13, 30], shape="tree"),
    dict(page=16, heads=1, group=2, dim=256, kv_lens=[90, 333], lengths=[1, 70]),
])
def test_float16_results_over_codes(dev, kind, case, monkeypatch):  # noqa: F811
    """The weights go in as two bfloat16 terms: the second is off by 2^-9 of what the first left over, 2^-9 of the weight.
    So the bound of 17 bits, 2^-18 of the weight, in place of the 7 that one term has."""
    log("case float16 results over %s dim %d" % (kind, case["dim"]))
    plain = D.attention
    monkeypatch.setattr(D, "attention", lambda q, k, v, seen, scale, weight, bits: plain(q, k, v, seen, scale, 17, bits))
    T.run_case(dev, kind, seed=21, given="fp16", **case)
