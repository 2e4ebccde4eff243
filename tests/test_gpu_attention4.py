"""The attention of a tree of tokens over a 4-bit cache: the checks of the other caches' tests, on caches in 4 bits.

A 4-bit cache's values are exact in bfloat16, so the oracle's bounds are those of a bfloat16 cache: one rounding of the
weights to 7 bits of fraction, or for float16 results to two such terms, 17 bits (the second is off by 2^-9 of what the
first left over).  And a weight below 2^-126 of the largest, the least normal float32, may count as nothing: 2^-126 |v| of
each position.  (A 4-bit value is often zero, so that the position with nearly all of the weight may add nothing and such
weights are all there is; in the other types they are lost in the rounding of its value.)"""
import numpy as np
import pytest

import test_gpu_tree_attention as T
from gpu_util import log
from oracle import decoding_oracle as D
from oracle import serving_oracle as S
from paper_2608_24658_amd import parason as PX
from serving_cases import Paged4
from test_gpu_tree_attention import dev  # noqa: F401

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def in_4_bits(monkeypatch):
    plain = D.attention
    monkeypatch.setattr(T, "Paged", Paged4)

    def attention(q, k, v, seen, scale, weight, bits):
        out, lse, out_tol, lse_tol = plain(q, k, v, seen, scale, 17 if bits == 10 else 7, bits)
        group, u = q.shape[1] // k.shape[1], np.nan_to_num(np.abs(v))
        size = np.einsum("np,phd->nhd", seen.astype(np.float64), u)
        out_tol = out_tol + 2.0 ** -126 * np.repeat(size, group, 1)
        if bits == 10:  # 65,504 is float16's largest, and from 65,520, half a step further, on results round to infinity
            out = np.where(np.abs(out) >= 65520, np.copysign(np.inf, out), out)
        return out, lse, out_tol, lse_tol

    monkeypatch.setattr(D, "attention", attention)


run_case = lambda dev, *a, **kw: T.run_case(dev, "fp4", *a, **kw)  # noqa: E731
GIVEN = pytest.mark.parametrize("given", ["bf16", "fp16"])


@GIVEN
@pytest.mark.parametrize("dim", [32, 64, 96, 128, 192, 256])
def test_single_tokens(dev, dim, given):  # noqa: F811
    log("case 4 bits single tokens dim %d %s" % (dim, given))
    kv = [1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129, 300]
    run_case(dev, 16, 2, 4, dim, kv, [1] * len(kv), seed=dim, given=given)


@pytest.mark.parametrize("heads,group", [(1, 1), (8, 1), (1, 16), (4, 7), (1, 48), (2, 40), (1, 130)])
def test_head_layouts(dev, heads, group):  # noqa: F811
    log("case 4 bits heads %d group %d" % (heads, group))
    run_case(dev, 32, heads, group, 64, [5, 70, 200], [1, 3, 2], seed=group)


@pytest.mark.parametrize("page", [1, 3, 8, 24, 64, 100, 256])
def test_pages(dev, page):  # noqa: F811
    log("case 4 bits pages of %d" % page)
    run_case(dev, page, 2, 2, 64, [1, page, page + 1, 3 * page - 1, 333], [1, 1, 1, min(3, 3 * page - 1), 40], seed=page,
             layout="slots" if page % 2 else "heads", pad=16 if page == 24 else 0)


@GIVEN
@pytest.mark.parametrize("lengths,before", [([100], [0]), ([257, 1, 64], [0, 30, 500]), ([33, 0, 129], [1000, 50, 1]), ([65], [63])])
def test_chains(dev, lengths, before, given):  # noqa: F811
    log("case 4 bits chain %s behind %s" % (lengths, before))
    run_case(dev, 16, 2, 4, 64, np.array(lengths) + before, lengths, seed=len(lengths), given=given)


@GIVEN
@pytest.mark.parametrize("dim", [32, 96, 128, 192, 256])
def test_chains_of_all_widths(dev, dim, given):  # noqa: F811
    log("case 4 bits chain dim %d" % dim)
    run_case(dev, 64, 1, 3, dim, [210, 90], [150, 90], seed=dim, given=given)
    run_case(dev, 24, 1, 5, dim, [310, 9], [10, 9], seed=dim + 1, given=given)
    run_case(dev, 24, 1, 3, dim, [310, 9], [10, 9], seed=dim + 1, given=given)


@GIVEN
@pytest.mark.parametrize("shape", ["chain", "star", "threads", "tree", "random", "empty"])
def test_trees(dev, shape, given):  # noqa: F811
    log("case 4 bits tree %s" % shape)
    run_case(dev, 16, 2, 3, 64, [8, 40, 100, 267, 1], [8, 13, 70, 3, 1], shape=shape, seed=5, given=given)
    run_case(dev, 24, 1, 4, 128, [300, 150], [150, 150], shape=shape, seed=6, given=given)
    run_case(dev, 16, 2, 4, 64, [700, 90, 64], [4, 8, 1], shape="tree", tree_lens=[640, 90, 64], seed=8, given=given)


def test_tokens_without_positions(dev):  # noqa: F811
    log("case 4 bits empty rows")
    out, lse = run_case(dev, 16, 2, 2, 64, [0, 3, 0], [2, 5, 0], seed=1)
    assert torch.all(out[1:3] == 0) and torch.all(lse[1:3] == -float("inf"))
    out, lse = run_case(dev, 16, 2, 2, 64, [6, 0], [6, 0], shape="empty", seed=2)
    assert torch.all(out[1:7:2] == 0) and torch.all(lse[1:7:2] == -float("inf"))


@GIVEN
def test_odd_strides(dev, given):  # noqa: F811
    log("case 4 bits odd strides")
    run_case(dev, 16, 2, 3, 64, [70, 300], [3, 200], odd=True, seed=3, given=given)
    run_case(dev, 16, 2, 3, 96, [70, 300], [1, 1], odd=True, seed=4, given=given)


@GIVEN
@pytest.mark.parametrize("lengths", [[4, 9], [90, 130]])
@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_what_is_not_seen_changes_nothing(dev, lengths, bad, given):  # noqa: F811
    """32 values of a head that hold a NaN or an infinity are NaN: for the tokens that see them."""
    log("case 4 bits masked %s %s" % (lengths, bad))
    rng = np.random.default_rng(1)

    def values(i, n):
        x = rng.standard_normal((2, n, 2, 64))
        at = n - 1 - rng.integers(0, min(n, lengths[i]), 3)
        x[1, at[0], :, 3] = bad
        x[1, at[1], 1, :] = -bad
        x[0, at[2], 0, 37] = bad
        return x

    for shape in (None, "tree", "empty"):
        run_case(dev, 16, 2, 4, 64, [lengths[0] + 37, lengths[1]], lengths, shape=shape, seed=11, values=values, given=given)


@GIVEN
@pytest.mark.parametrize("lengths", [[4, 9], [40, 60]])
def test_scales_that_a_write_does_not_make(dev, lengths, given):  # noqa: F811
    """Scale bytes of 253 and 254, whose larger values are infinities, and 255, in values of positions that some tokens
    see and others do not: the smaller values of the same 32 count as they are, those of other 32s too."""
    log("case 4 bits infinite scales %s %s" % (lengths, given))
    rng = np.random.default_rng(2)

    def spoil(P, seens):
        for i, n in enumerate(lengths):
            for byte, back, at in ((253, 1, 0), (254, 2, 1), (255, 3, 0)):
                pos = int(P.kv_lens[i]) - back
                pg, slot = (int(v) for v in P.place(i, pos))
                codes = rng.integers(0, 16, 32).astype(np.uint8)
                P.cache.v.view(torch.uint8)[pg, slot, 1, 16 * at: 16 * at + 16] = torch.from_numpy(S.pack4(codes)).to(dev)
                P.cache.v_scale.view(torch.uint8)[pg, slot, 1, at] = byte
                P.held[i][1][pos, 1, 32 * at: 32 * at + 32] = S.values4(codes, np.array([byte], np.uint8))

    for shape in (None, "tree"):
        run_case(dev, 16, 2, 4, 64, [lengths[0] + 37, lengths[1]], lengths, shape=shape, seed=12, given=given, spoil=spoil)


@GIVEN
def test_large_and_small_scores(dev, given):  # noqa: F811
    log("case 4 bits scores")
    big = lambda i, n: np.random.default_rng(i).standard_normal((2, n, 1, 64)) * np.array([30.0, 1.0])[:, None, None, None]  # noqa: E731
    run_case(dev, 16, 1, 4, 64, [200, 90], [1, 60], values=big, scale=1.0, seed=2, given=given)
    run_case(dev, 16, 1, 4, 64, [200, 90], [1, 60], values=big, scale=-0.5, seed=2, given=given)
    run_case(dev, 16, 1, 4, 64, [200, 90], [1, 60], scale=0.0, seed=2, given=given)


def test_long_rows(dev):  # noqa: F811
    """Rows cut into parts, for every width of a block of columns."""
    log("case 4 bits long rows")
    run_case(dev, 64, 2, 2, 64, [9000, 4001, 17], [1, 1, 1], seed=4)
    run_case(dev, 16, 1, 4, 128, [6000], [5], shape="tree", seed=5)
    run_case(dev, 16, 1, 16, 64, [5000, 100], [9, 7], seed=6)
    lengths = [150, 1, 3, 1, 0, 2, 1, 40]
    run_case(dev, 64, 2, 2, 64, [9100, 1, 300, 4097, 0, 2049, 1025, 5000], lengths, seed=7)
    run_case(dev, 64, 2, 2, 64, [9100, 1, 300, 4097, 0, 2049, 1025, 5000], lengths, shape="threads", seed=8)


@GIVEN
@pytest.mark.parametrize("dim", [64, 128, 256])
def test_ragged_rows(dev, dim, given):  # noqa: F811
    """Rows of all lengths: some without tokens or positions, long ones that several blocks share, trees, and several
    blocks of columns."""
    log("case 4 bits ragged dim %d %s" % (dim, given))
    kv = [3000, 0, 1, 128, 129, 5000, 40, 700, 0, 513, 4096, 77]
    run_case(dev, 16, 2, 4, dim, kv, [1, 1, 1, 0, 1, 1, 0, 1, 0, 1, 1, 1], seed=3, given=given)
    run_case(dev, 24, 1, 4, dim, kv, [3, 2, 1, 0, 5, 4, 0, 12, 0, 1, 3, 2], seed=4, given=given)
    run_case(dev, 24, 1, 4, dim, [max(k, 9) for k in kv], [9, 2, 1, 0, 5, 4, 0, 9, 0, 1, 3, 2], shape="tree", seed=5, given=given)
    run_case(dev, 64, 8, 4, dim, [600] * 40, [1] * 40, seed=6, given=given)


def test_long_rows_that_are_bad(dev):  # noqa: F811
    """Bad rows, pages and trees among rows that are cut into parts."""
    log("case 4 bits long bad rows")
    P = Paged4(dev, [3000] * 6, 8, 2, 64, "fp4", seed=3)
    rng = np.random.default_rng(0)
    P.fill(lambda i, n: rng.standard_normal((2, n, 2, 64)))
    rows, total, _ = P.rows([2] * 6)
    kv, pages, st = rows.kv_lens.clone(), rows.pages.clone(), rows.starts.clone()
    kv[1], st[3], pages[4, 200] = 3001, -1, P.n_pages
    rows = rows._replace(kv_lens=kv, pages=pages, starts=st)
    q = torch.randn(total, 4, 64, device=dev, dtype=torch.bfloat16)
    status, out = torch.zeros(6, dtype=torch.int32, device=dev), torch.full_like(q, 3.0)
    PX.tree_attention(q, P.cache, rows, out=out, status=status)
    assert status.cpu().tolist() == [0, PX.KV_BAD_ROW, 0, PX.KV_BAD_ROW, PX.KV_BAD_PAGE, 0]
    got = out.cpu().double()
    assert torch.isnan(got[2:4]).all() and (got[6:8] == 3.0).all() and torch.isnan(got[8:10]).all()
    for i in (0, 2, 5):
        o, _, tol, _ = D.attention(q[2 * i: 2 * i + 2].cpu().double().numpy(), *P.held[i], D.visible(3000, 2), 0.125, 7, 7)
        assert np.all(np.abs(got[2 * i: 2 * i + 2].numpy() - o) <= tol)
    # trees that their masks do not hold, and none of whose words are read
    rows, total, _ = P.rows([2] * 6)
    mask = torch.full((total, 1), -1, dtype=torch.int64, device=dev)
    trees = torch.tensor([2, 40, 65, -1, 2 ** 31 - 1, 0], dtype=torch.int32, device=dev)
    status.zero_()
    got, lse = PX.tree_attention(q, P.cache, rows, mask=mask, tree_lens=trees, status=status, lse=True)
    b = PX.KV_BAD_ROW
    assert status.cpu().tolist() == [0, 0, b, b, b, 0]
    assert torch.isnan(got[4:10]).all() and torch.isnan(lse[4:10]).all() and torch.isfinite(got[:4]).all() and torch.isfinite(got[10:]).all()
    # a pool without pages
    none = PX.KVCache(*(t[:0] for t in P.cache))
    got = PX.tree_attention(q, none, rows)
    assert torch.isnan(got).all()


def test_growing_rows_in_a_graph(dev):  # noqa: F811
    """Captured, and replayed over rows that have grown meanwhile; two graphs with workspaces of their own."""
    log("case 4 bits graph")
    P = Paged4(dev, [3000, 900, 2000], 16, 2, 64, "fp4", seed=3)
    rng = np.random.default_rng(0)
    P.fill(lambda i, n: rng.standard_normal((2, n, 2, 64)))
    rows, total, _ = P.rows([1] * 3)
    q = torch.randn(total, 8, 64, device=dev, dtype=torch.bfloat16)
    ws = [torch.empty(PX.tree_attention_workspace_size(P.cache, rows, total, 8), dtype=torch.uint8, device=dev) for _ in range(2)]
    outs, graphs = [torch.empty_like(q) for _ in range(2)], []
    torch.cuda.synchronize()
    for w, o in zip(ws, outs):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            PX.tree_attention(q, P.cache, rows, out=o, workspace=w)
        graphs.append(g)
    for lens in ([3000, 900, 2000], [1, 900, 0], [2500, 17, 1999]):
        rows.kv_lens.copy_(torch.tensor(lens, dtype=torch.int32))
        want = PX.tree_attention(q, P.cache, rows)
        for g, o, w in zip(graphs, outs, ws):
            o.fill_(7), w.fill_(0xFF)
            (torch.randn(1000, device=dev) * 2).sum().item()
            g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(o, want) for o in outs)
        for i, n in enumerate(lens):
            o, _, tol, _ = D.attention(q[i: i + 1].cpu().double().numpy(), *(x[:n] for x in P.held[i]), D.visible(n, 1), 0.125, 7, 7)
            assert np.all(np.abs(want[i: i + 1].cpu().double().numpy() - o) <= tol)


@GIVEN
@pytest.mark.parametrize("kv_lens,lengths,group", [([9000, 4001, 513, 63], [1, 1, 1, 1], 4), ([9100, 2049, 31], [3, 4, 3], 8),
                                                   ([9100, 5000, 1, 4097], [150, 40, 1, 2], 2), ([33000], [1], 4)])
def test_every_position_counts_once(dev, given, kv_lens, lengths, group):  # noqa: F811
    """Keys of zero, and as values one one among zeros, in dimension position % 256: result d times the number of
    positions seen is the number of those that belong to d, some tens.  One position more or less changes it by 1 / 130 or
    more; the weights are equal powers of two, the values exact, so what is off is the sum (kv additions, 2^-24 each) and
    the result's rounding (2^-9): 1 / 170 at most."""
    log("case 4 bits every position once kv %s tokens %s" % (kv_lens, lengths))
    dim = 256
    P = Paged4(dev, kv_lens, 24, 1, dim, "fp4", seed=2)

    def values(i, n):
        x = np.zeros((2, n, 1, dim))
        x[1, np.arange(n), 0, np.arange(n) % dim] = 1.0
        return x

    P.fill(values)
    rows, total, starts = P.rows(lengths)
    q = torch.as_tensor(np.random.default_rng(0).standard_normal((total, group, dim)).astype(np.float32)).to(T.torch_type(given))
    out, lse = PX.tree_attention(q.to(dev), P.cache, rows, lse=True)
    out, lse = out.cpu().double().numpy(), lse.cpu().double().numpy()
    for i, n in enumerate(lengths):
        for j in range(n):
            seen = kv_lens[i] - n + j + 1
            want = np.bincount(np.arange(max(seen, 0)) % dim, minlength=dim) * 1.0
            if seen <= 0:
                assert np.all(out[starts[i] + j] == 0)
                continue
            for h in range(group):
                assert np.all(np.abs(out[starts[i] + j, h] * seen - want) <= want / 170), (i, j, h)
                assert abs(lse[starts[i] + j, h] - np.log(seen)) <= (seen + 16) * 2.0 ** -24 * max(1.0, np.log(seen))


def test_scales_of_all_sizes(dev):  # noqa: F811
    """Groups of a head whose scales lie far apart, beyond what float16 holds: each counts as it is."""
    log("case 4 bits scales")
    rng = np.random.default_rng(4)

    def values(i, n):
        e = rng.integers(-30, 31, (2, n, 1, 4)).repeat(32, -1)
        x = rng.standard_normal((2, n, 1, 128)) * 2.0 ** e
        x[0] *= 2.0 ** -30  # scores that leave several positions a weight
        return x

    for given in ("bf16", "fp16"):
        # (float16 results do not hold values of 2^30; the ones here are smaller by the choice of the second scale)
        v = values if given == "bf16" else (lambda i, n: values(i, n) * np.array([1.0, 2.0 ** -20])[:, None, None, None])
        run_case(dev, 16, 1, 4, 128, [90, 200, 300], [1, 3, 70], seed=3, values=v, given=given, scale=0.5)


def test_queries_of_float16(dev):  # noqa: F811
    """All 11 bits of a float16 query count: keys of one value, a query whose last bit decides."""
    log("case 4 bits float16 queries")
    P = Paged4(dev, [2], 16, 1, 32, "fp4", seed=0)
    x = np.zeros((2, 2, 1, 32))
    x[0, 0, 0, 0] = 6.0
    x[1, 0], x[1, 1] = 1.0, -1.0
    P.fill(lambda i, n: x)
    rows, _, _ = P.rows([1])
    q = torch.zeros(1, 2, 32, dtype=torch.float16)
    q[0, 0, 0], q[0, 1, 0] = 2047.0 / 1024, 2046.0 / 1024
    _, lse = PX.tree_attention(q.to(dev), P.cache, rows, scale=1.0, lse=True)
    want = np.log(np.exp(6.0 * np.array([2047, 2046]) / 1024) + 1)
    assert np.abs(lse.cpu().double().numpy()[0] - want).max() < 1e-5


def test_rows_and_pages_that_are_bad(dev):  # noqa: F811
    log("case 4 bits bad rows")
    P = Paged4(dev, [40] * 4, 8, 2, 64, "fp4", seed=3)
    rng = np.random.default_rng(0)
    P.fill(lambda i, n: rng.standard_normal((2, n, 2, 64)))
    for n in (2, 33):
        rows, total, starts = P.rows([n] * 4)
        kv, pages = rows.kv_lens.clone(), rows.pages.clone()
        kv[1] = 41
        pages[2, 3] = P.n_pages
        rows = rows._replace(kv_lens=kv, pages=pages)
        q = torch.randn(total, 4, 64, device=dev, dtype=torch.bfloat16)
        status = torch.zeros(4, dtype=torch.int32, device=dev)
        got, lse = PX.tree_attention(q, P.cache, rows, lse=True, status=status)
        assert status.cpu().tolist() == [0, PX.KV_BAD_ROW, PX.KV_BAD_PAGE, 0]
        got = got.cpu().double()
        assert torch.isnan(got[n: 2 * n]).all() and torch.isnan(got[3 * n - 1]).all()
        for i in (0, 3):
            at = slice(i * n, i * n + n)
            o, _, tol, _ = D.attention(q[at].cpu().double().numpy(), *P.held[i], D.visible(40, n), 0.125, 7, 7)
            assert np.all(np.abs(got[at].numpy() - o) <= tol)


def test_values_are_those_of_a_16_bit_cache(dev):  # noqa: F811
    """What kv_read gives, put into a bfloat16 cache, attends alike: the same operands of the same products, so equal
    results but for the order of the sums (2^-22 of float32 sums) and a rounding of each result that this may tip."""
    log("case 4 bits against 16")
    rng = np.random.default_rng(0)
    P = Paged4(dev, [700, 90], 16, 2, 128, "fp4", seed=1)
    P.fill(lambda i, n: rng.standard_normal((2, n, 2, 128)))
    B = T.__dict__["Paged"].__mro__[1](dev, [700, 90], 16, 2, 128, "bf16", 1)
    B.fill(lambda i, n: np.stack(P.held[i]))
    for lengths in ([1, 1], [90, 70]):
        rows, total, _ = P.rows(lengths)
        q = torch.randn(total, 8, 128, device=dev, dtype=torch.bfloat16)
        a, za = PX.tree_attention(q, P.cache, rows, lse=True)
        b, zb = PX.tree_attention(q, B.cache, B.rows(lengths)[0], lse=True)
        assert (za - zb).abs().max() < 1e-5
        assert (a.float() - b.float()).abs().max() <= 2.0 ** -7 * b.float().abs().max()
    assert S.GRID4[-1] == 6.0
