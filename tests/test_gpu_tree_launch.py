"""Calls whose grids, by their bounds, have more threads than one launch takes (2^32 - 1)."""
import numpy as np
import pytest

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


def ragged(dev, lengths, kv_lens, bound, heads, q_heads, dim=16, page=64, seed=0):
    """bfloat16 rows whose longest may have `bound` tokens: queries, the cache, the rows, and what each row holds."""
    rng = np.random.default_rng(seed)
    lengths, kv_lens = np.asarray(lengths), np.asarray(kv_lens)
    need = -(-kv_lens // page)
    pages = np.zeros((len(lengths), int(need.max())), np.int32)
    pages[np.arange(pages.shape[1])[None, :] < need[:, None]] = rng.permutation(int(need.sum()))
    gen = torch.Generator(device=dev).manual_seed(seed)
    kv = [torch.randn(int(need.sum()), page, heads, dim, generator=gen, device=dev).bfloat16() for _ in "kv"]
    q = torch.randn(int(lengths.sum()), q_heads, dim, generator=gen, device=dev).bfloat16()
    starts = np.cumsum(lengths) - lengths
    put = lambda a, dt: torch.as_tensor(a).to(device=dev, dtype=dt)  # noqa: E731
    rows = PX.KVRows(put(starts, torch.int64), put(lengths, torch.int32), put(kv_lens, torch.int32), put(pages, torch.int32), bound,
                     int(kv_lens.max()))

    def held(i):
        at = np.arange(kv_lens[i])
        return [x[put(pages[i, at // page], torch.int64), put(at % page, torch.int64)].double().cpu().numpy() for x in kv]

    return q, PX.KVCache(*kv), rows, starts, held


def check_tokens(q, out, lse, held, starts, lengths, kv_lens, tokens):
    for i, j in tokens:
        seen = D.visible(int(kv_lens[i]), int(lengths[i]))[j: j + 1] if lengths[i] < 100 else \
            (np.arange(kv_lens[i]) <= kv_lens[i] - lengths[i] + j)[None, :]
        t = int(starts[i] + j)
        o, z, tol, ztol = D.attention(q[t: t + 1].cpu().double().numpy(), *held(i), seen, q.shape[2] ** -0.5, 7, 7)
        assert np.all(np.abs(out[t: t + 1].cpu().double().numpy() - o) <= tol), (i, j)
        assert np.all(np.abs(lse[t: t + 1].cpu().double().numpy() - z) <= ztol), (i, j)


def test_few_tokens_under_a_large_bound(dev):
    """A hundred rows of a token each that may have 21,000: their parts' results are joined, too."""
    log("case few tokens, bound 21000")
    lengths, kv_lens = [1] * 100, [40 + 50 * (i % 7) + (9000 if i == 3 else 0) for i in range(100)]
    q, cache, rows, starts, held = ragged(dev, lengths, kv_lens, 21000, 8, 32)
    status = torch.zeros(100, dtype=torch.int32, device=dev)
    out, lse = PX.tree_attention(q, cache, rows, out=torch.full_like(q, 9.0), lse=True, status=status)
    assert not status.any()
    check_tokens(q, out, lse, held, starts, lengths, kv_lens, [(i, 0) for i in range(100)])


def test_a_prompt_among_a_thousand_tokens(dev):
    """One prompt of 32,768 tokens and 1,023 single ones, 64 query heads over 8: 2^24 blocks of 256 threads."""
    log("case 32768 tokens among 1023 rows of one")
    lengths, kv_lens = [1] * 1024, [1 + 37 * i % 290 for i in range(1024)]
    lengths[700], kv_lens[700] = 32768, 32768
    q, cache, rows, starts, held = ragged(dev, lengths, kv_lens, 32768, 8, 64)
    status = torch.zeros(1024, dtype=torch.int32, device=dev)
    out, lse = PX.tree_attention(q, cache, rows, out=torch.full_like(q, 9.0), lse=True, status=status)
    assert not status.any()
    check_tokens(q, out, lse, held, starts, lengths, kv_lens,
                 [(i, 0) for i in range(0, 1024, 31)] + [(1023, 0), (700, 0), (700, 1), (700, 15000), (700, 32767)])
    # (of the tokens not looked at above, too, every one has its result)
    assert torch.isfinite(lse).all() and not (out == 9.0).all(-1).any()
