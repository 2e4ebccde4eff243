"""Beam selection and reordering on the GPU against the oracle in 64 bits.

Scores: the oracle's within 2^-14 (a float32 sum of up to 2^10 exponentials a lane, 2^-24 each, and of the lanes) and
half an ulp of the float that is stored.  The choice: exact where the candidates are further apart than that or
exactly equal (the tests below with ties); otherwise every chosen candidate has the score of its place."""
import numpy as np
import pytest

from gpu_util import log
from oracle import decoding_oracle as D
from paper_2608_24658_amd import parason as PX

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


@pytest.fixture(scope="module")
def dev():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    return torch.device("cuda:0")


def states_of(flags, dev):
    s = np.zeros((len(flags), 4), np.int32)
    s[:, 3] = flags
    return torch.as_tensor(s).to(dev).view(torch.uint8).reshape(-1)


def check(logits, scores, flags, beams, out, vocab, exact=False):
    cand = D.beam_candidates(logits.float().cpu().numpy(), scores, flags, beams)
    place = D.beam_select(cand, beams)
    groups = cand.shape[0]
    score, parent, token = (out[k].cpu().numpy().reshape(groups, beams) for k in ("score", "parent", "token"))
    rows = np.arange(groups * beams).reshape(groups, beams)
    none = place < 0
    assert np.array_equal(parent[none], rows[none]) and np.all(token[none] == -1) and np.all(score[none] == -np.inf)
    want = np.where(none, -np.inf, np.take_along_axis(cand, np.maximum(place, 0), 1))
    tol = 2.0 ** -14 + np.abs(np.where(none, 0, want)) * 2.0 ** -23
    assert np.all(np.abs(score[~none].astype(np.float64) - want[~none]) <= tol[~none])
    got = np.where(none, -1, (parent - rows[:, :1]) * (vocab + 1) + token + 1)
    if exact:
        assert np.array_equal(got, place), (got[got != place][:5], place[got != place][:5])
        return
    for g in range(groups):
        live = got[g][~none[g]]
        assert len(set(live.tolist())) == live.size
        c = cand[g][live]
        assert np.all(np.abs(c - want[g][~none[g]]) <= 2 * tol[g][~none[g]]), g
        # equal candidates of one row: in order, the lowest first
        for a, b in zip(live[:-1], live[1:]):
            if cand[g][a] == cand[g][b] and a // (vocab + 1) == b // (vocab + 1):
                assert a < b
        last = cand[g][live[-1]] if live.size else 0
        for a in live:
            same = np.nonzero(cand[g] == cand[g][a])[0]
            same = same[(same // (vocab + 1) == a // (vocab + 1)) & (same < a)]
            assert np.isin(same, live).all() or cand[g][a] > last


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("groups,beams,vocab", [(1, 1, 1), (3, 1, 50), (2, 4, 3), (5, 3, 1000), (2, 8, 4099), (1, 64, 700), (1, 33, 20001),
                                               (2, 4, 151936), (300, 2, 257)])
def test_select(dev, dtype, groups, beams, vocab):
    log("case beam %s %dx%d vocab %d" % (dtype, groups, beams, vocab))
    rng = np.random.default_rng(beams * vocab + groups)
    rows = groups * beams
    x = torch.as_tensor((rng.standard_normal((rows, vocab)) * 3).astype(np.float32)).to(TYPES[dtype])
    x[torch.as_tensor(rng.random((rows, vocab)) < 0.1)] = float("-inf")
    scores = (-20 * rng.random(rows)).astype(np.float32)
    flags = np.where(rng.random(rows) < 0.15, rng.integers(1, 4, rows), 0)
    if groups > 1:
        scores[:beams] = np.where(np.arange(beams) > 0, -np.inf, -1.5)  # a prompt that has just begun
        flags[:beams] = 0
    wide = torch.full((rows, vocab + 5), float("inf"), dtype=TYPES[dtype], device=dev)
    view = wide[:, 1: vocab + 1]
    view.copy_(x)
    out = PX.beam_select(view, torch.as_tensor(scores).to(dev), beams, states=states_of(flags, dev))
    check(x, scores, flags, beams, out, vocab)
    out = PX.beam_select(x.to(dev), torch.as_tensor(scores).to(dev), beams)
    check(x, scores, flags * 0, beams, out, vocab)


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("vocab", [7, 640, 30001])
def test_ties(dev, dtype, vocab):
    """Equal logits, equal rows: the lowest row and token first.  All logits of a row equal; few values; one row twice."""
    log("case ties %s vocab %d" % (dtype, vocab))
    rng = np.random.default_rng(vocab)
    beams = 6
    x = np.zeros((4 * beams, vocab), np.float32)
    x[beams: 2 * beams] = rng.integers(-3, 3, vocab)[None, :]           # the same row six times
    x[2 * beams: 3 * beams] = 8.0 * rng.integers(0, 2, vocab)[None, :]  # two values
    x[3 * beams:] = -np.inf
    x[3 * beams:, vocab // 2] = 1.0                                     # one token each
    t = torch.as_tensor(x).to(TYPES[dtype])
    scores = np.zeros(4 * beams, np.float32)
    out = PX.beam_select(t.to(dev), torch.as_tensor(scores).to(dev), beams)
    check(t, scores, np.zeros(4 * beams, int), beams, out, vocab, exact=True)
    # the beams of a fresh prompt: one row counts
    scores[1:beams] = -np.inf
    out = PX.beam_select(t.to(dev), torch.as_tensor(scores).to(dev), beams)
    check(t, scores, np.zeros(4 * beams, int), beams, out, vocab, exact=True)


def test_rows_that_offer_nothing(dev):
    """NaN, +inf, nothing but -inf, a NaN score, errors, finished rows; a group with nothing at all."""
    log("case rows that offer nothing")
    beams, vocab = 4, 5000
    rng = np.random.default_rng(0)
    x = (rng.standard_normal((5 * beams, vocab)) * 2).astype(np.float32)
    scores = np.linspace(-1, -9, 5 * beams).astype(np.float32)
    flags = np.zeros(5 * beams, int)
    x[0, 17], x[1, 4999], x[2] = np.nan, np.inf, -np.inf
    scores[4], scores[5], scores[6] = np.nan, np.inf, -np.inf
    flags[8:12] = [2, 1, 3, 2]
    flags[12:16] = 1
    x[16:] = np.nan
    x[17] = -np.inf
    out = PX.beam_select(torch.as_tensor(x).to(dev), torch.as_tensor(scores).to(dev), beams, states=states_of(flags, dev))
    check(torch.as_tensor(x), scores, flags, beams, out, vocab)
    assert out["token"].cpu().tolist()[8:12] == [-1] * 4 and out["parent"].cpu().tolist()[8:12] == [8, 11, 10, 11]
    assert out["score"].cpu().tolist()[12:] == [-np.inf] * 8


def test_few_tokens_left(dev):
    """Rows that decode_step has left three tokens of: fewer candidates than beams."""
    log("case few tokens")
    beams, vocab = 16, 2000
    rng = np.random.default_rng(3)
    x = np.full((2 * beams, vocab), -np.inf, np.float32)
    for r in range(2 * beams):
        at = rng.choice(vocab, 3, replace=False)
        x[r, at] = rng.standard_normal(3)
    scores = np.full(2 * beams, -np.inf, np.float32)
    scores[[0, beams, beams + 1, beams + 9]] = [0.0, -1.0, -2.0, -0.5]
    out = PX.beam_select(torch.as_tensor(x).to(dev), torch.as_tensor(scores).to(dev), beams)
    check(torch.as_tensor(x), scores, np.zeros(2 * beams, int), beams, out, vocab)
    assert np.isfinite(out["score"].cpu().numpy()).sum() == 3 + 9


@pytest.mark.parametrize("rows", [1, 7, 500])
def test_reorder(dev, rows):
    """Every kind of row: 16-byte states, odd byte counts, strided rows, long rows; parents outside leave dst alone."""
    log("case reorder %d" % rows)
    rng = np.random.default_rng(rows)
    parent = rng.integers(0, rows, rows).astype(np.int32)
    arrays = [
        torch.randint(0, 255, (rows * 16,), dtype=torch.uint8),
        torch.randint(-9, 9, (rows, 301), dtype=torch.int32),
        torch.randint(0, 255, (rows, 7), dtype=torch.uint8),
        torch.randn(rows, 3, 50),
        torch.randint(-2 ** 62, 2 ** 62, (rows, 5000), dtype=torch.int64),
        torch.randn(rows).to(torch.bfloat16),
        torch.empty(rows, 0),
        torch.randn(rows, 40, 3).to(torch.float16)[:, :21],
    ]
    d = [a.to(dev) for a in arrays]
    d[7] = torch.zeros(rows, 40, 3, dtype=torch.float16, device=dev)[:, :21]
    d[7].copy_(arrays[7])
    out = PX.beam_reorder(torch.as_tensor(parent).to(dev), d)
    for a, o in zip(arrays, out):
        want = a.reshape(rows, -1)[torch.as_tensor(parent).long()].reshape(o.shape) if a.numel() else a
        assert torch.equal(o.cpu(), want)
    # into views at odd addresses, with parents that name no row
    parent[:: 3] = -1
    if rows > 5:
        parent[1] = rows
    src = torch.randint(0, 255, (rows, 133), dtype=torch.uint8, device=dev)[:, 1:132]
    dst = torch.full((rows, 150), 9, dtype=torch.uint8, device=dev)
    PX.beam_reorder(torch.as_tensor(parent).to(dev), [src], out=[dst[:, 3:134]])
    want = torch.full((rows, 150), 9, dtype=torch.uint8)
    ok = (parent >= 0) & (parent < rows)
    want[torch.as_tensor(ok), 3:134] = src.cpu()[torch.as_tensor(parent[ok]).long()]
    assert torch.equal(dst.cpu(), want)


def test_scores_in_place_and_in_a_graph(dev):
    """The new scores over the old ones, and a graph replayed with other work between the replays."""
    log("case beam graph")
    x = torch.randn(8, 30000, device=dev)
    scores = -torch.rand(8, device=dev)
    want = PX.beam_select(x, scores, 4)
    keep = scores.clone()
    parent, token = torch.empty(2, 8, dtype=torch.int32, device=dev)
    ws = torch.empty(PX.beam_workspace_size(2, 4, 30000), dtype=torch.uint8, device=dev)

    def call():
        rc = PX.lib().parason_beam_select(x.data_ptr(), 30000, 30000, PX.DTYPE_F32, scores.data_ptr(), None, 2, 4, scores.data_ptr(),
                                          parent.data_ptr(), token.data_ptr(), ws.data_ptr(), ws.numel(),
                                          torch.cuda.current_stream().cuda_stream)
        assert rc == PX.OK

    call()
    torch.cuda.synchronize()
    assert torch.equal(scores, want["score"]) and torch.equal(parent, want["parent"]) and torch.equal(token, want["token"])
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        call()
    for _ in range(3):
        scores.copy_(keep)
        ws.fill_(0xFF)
        token.zero_()
        torch.randn(1000, device=dev).sum().item()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(scores, want["score"]) and torch.equal(parent, want["parent"]) and torch.equal(token, want["token"])
