"""Which beams beam_select chooses, exactly: the largest float32 scores, as returned, equal ones to the lowest row and
token.  The logits are such that a row's ln sum is known to the last bit, or that its last bit does not matter: one token
that outweighs the others beyond float32, sums far enough from the middle between two floats, or equal logits."""
import numpy as np
import pytest

from gpu_util import log
from oracle import decoding_oracle as D
from paper_2608_24658_amd import parason as PX
from test_gpu_beam import TYPES, dev, states_of  # noqa: F401

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

NONE = np.float32(-np.inf)


def select(dev, x, scores, beams, flags=None, lse=None):  # noqa: F811
    """The choice on the GPU and the oracle's: (score, place in the group), -1 where there is none."""
    rows, vocab = x.shape
    s = None if flags is None else states_of(flags, dev)
    out = PX.beam_select(x.to(dev), torch.as_tensor(scores).to(dev), beams, states=s)
    score, parent, token = (out[k].cpu().numpy().reshape(-1, beams) for k in ("score", "parent", "token"))
    first = np.arange(0, rows, beams)[:, None]
    # returned scores never rise, and equal ones are in the order of row and token
    here = (parent - first).astype(np.int64) * (vocab + 1) + token + 1
    live = score > NONE
    assert np.all(np.diff(live.astype(int), axis=1) <= 0)
    a, b, both = score[:, :-1], score[:, 1:], live[:, 1:]
    assert np.all((a >= b)[both]) and np.all((here[:, :-1] < here[:, 1:])[both & (a == b)])
    cand = D.beam_scores(x.float().numpy(), scores, np.zeros(rows, int) if flags is None else flags, beams, lse=lse)
    place = D.beam_select(cand, beams)
    want = np.where(place < 0, NONE, np.take_along_axis(cand, np.maximum(place, 0), 1))
    return score, np.where(live, here, -1), want, place


def same(got):
    score, here, want, place = got
    assert np.array_equal(here, place), (here[here != place][:6], place[here != place][:6])
    assert np.array_equal(score, want)


@pytest.mark.parametrize("dtype,base,spread", [("f32", -3000.0, 0.05), ("f32", -3e5, 2.0), ("f16", -1.2e6, 4.0), ("bf16", -1.2e7, 30.0)])
@pytest.mark.parametrize("groups,beams,vocab", [(5, 4, 700), (4, 8, 20001), (2, 32, 9000), (1, 64, 30001)])
def test_scores_that_rounding_makes_equal(dev, dtype, base, spread, groups, beams, vocab):  # noqa: F811
    """Different logits of a row whose float32 scores are equal, thousands of them, over several chunks: the lowest token
    counts, not the largest logit.  One to three rows of a group have a score, a float32 apart or equal."""
    log("case equal after rounding %s base %g %dx%d vocab %d" % (dtype, base, groups, beams, vocab))
    rng = np.random.default_rng(beams * vocab)
    rows = groups * beams
    x = torch.as_tensor((-120 - spread * rng.random((rows, vocab))).astype(np.float32)).to(TYPES[dtype])
    x[torch.arange(rows), torch.as_tensor(rng.integers(0, vocab, rows))] = 0.0
    scores = np.full(rows, -np.inf, np.float32)
    for g in range(groups):
        for k in range(min(beams, 1 + g % 3)):
            scores[g * beams + (k * 5) % beams] = np.float32(base) if k != 1 else np.nextafter(np.float32(base), np.float32(0))
    same(select(dev, x, scores, beams))


@pytest.mark.parametrize("beams,vocab", [(1, 700), (1, 20001), (3, 9000)])
def test_the_lowest_of_a_rows_first(dev, beams, vocab):  # noqa: F811
    """The best float32 score of a row belongs to many tokens with different logits: a row that is nearly flat, and scores
    near -1e6, which come in steps of 1/16.  Rows whose choice another unit in the last place of ln sum would not change."""
    log("case flat rows %d vocab %d" % (beams, vocab))
    rng = np.random.default_rng(vocab)
    rows, base, made = 4 * beams, np.float32(-1e6), []
    while len(made) < rows:
        x = (2.0 ** -12 * rng.integers(0, 400, vocab)).astype(np.float32)
        lse = D.beam_lse(x)[1]
        near = [base + (x - np.float32(lse + k * np.spacing(lse))) for k in (-2, 0, 2)]
        if np.array_equal(near[0], near[1]) and np.array_equal(near[1], near[2]):
            made.append(x)
    same(select(dev, torch.as_tensor(np.stack(made)), np.full(rows, base), beams))


def far_from_middles(row):
    """Whether a row's top + ln sum lies 2^-19 or more from the middle of two float32 values: a float32 sum of up to eight
    exponentials a thread and the wave's threads (18 roundings in all, 2^-24 each, of the sum and so of its logarithm) and
    a float32 logarithm below 8 (2^-21) then leave the rounded value as it is."""
    exact, rounded = D.beam_lse(row)
    step = float(np.spacing(np.float32(rounded)))
    return abs(exact / step - np.floor(exact / step) - 0.5) * step >= 2.0 ** -19


@pytest.mark.parametrize("dtype,steps,step", [("f32", 2048, 2.0 ** -10), ("f16", 32, 2.0 ** -4), ("bf16", 4, 0.5)])
@pytest.mark.parametrize("seed", range(4))
def test_rows_a_float_apart(dev, dtype, steps, step, seed):  # noqa: F811
    """Rows that hold the same logits in another order, and scores that are equal or neighbouring floats: candidates of
    different rows are equal or one unit in the last place apart, and a row's ln sum must not depend on its order."""
    log("case rows a float apart %s seed %d" % (dtype, seed))
    rng = np.random.default_rng(100 + seed)
    groups, beams, vocab = 6, 8, 2000
    kinds = []
    while len(kinds) < 2 * groups:
        row = 100 - step * rng.integers(0, steps, vocab)
        row[0] = 100
        if far_from_middles(row):
            kinds.append(row)
    x = np.stack([rng.permutation(kinds[2 * g + (b >= 5)]) for g in range(groups) for b in range(beams)])
    scores = np.full(groups * beams, -37.3, np.float32)
    for r in range(scores.size):
        for _ in range(int(rng.integers(0, 3))):
            scores[r] = np.nextafter(scores[r], np.float32(0))
    t = torch.as_tensor(x.astype(np.float32)).to(TYPES[dtype])
    assert np.array_equal(t.double().numpy(), x)
    same(select(dev, t, scores, beams))


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("groups,beams,vocab", [(2, 32, 20001), (2, 64, 700), (1, 64, 30001)])
def test_more_equal_candidates_than_a_list_holds(dev, dtype, groups, beams, vocab):  # noqa: F811
    """Every logit equal and every score equal: beams * beams candidates of every chunk; then with finished rows of the
    same score, rows in error and rows without a score among them."""
    log("case all equal %s %dx%d vocab %d" % (dtype, groups, beams, vocab))
    rows = groups * beams
    x = torch.zeros(rows, vocab, dtype=TYPES[dtype])
    # ln sum as the library has it (the logarithm of a whole number: a float32 logarithm's unit in the last place)
    lse = -PX.beam_select(x[:1].to(dev), torch.zeros(1, device=dev), 1)["score"].cpu().numpy()[0]
    assert abs(float(lse) - np.log(vocab)) <= float(np.spacing(lse))
    lses = np.full(rows, lse, np.float32)
    scores = np.full(rows, -5.0, np.float32)
    same(select(dev, x, scores, beams, lse=lses))
    rng = np.random.default_rng(vocab)
    flags = np.where(rng.random(rows) < 0.1, rng.integers(1, 3, rows), 0)
    scores[flags == 2] = np.float32(-5) + (np.float32(0) - lse)
    scores[rng.random(rows) < 0.2] = -np.inf
    same(select(dev, x, scores, beams, flags, lse=lses))
    # a row without candidates, and one of three that is better than the rest
    b = beams // 2
    scores[b], flags[b] = -4.0, 0
    x[1] = x[b] = float("-inf")
    x[b, vocab // 2: vocab // 2 + 3] = 1.0
    lses[b] = -PX.beam_select(x[b: b + 1].to(dev), torch.zeros(1, device=dev), 1)["score"].cpu().numpy()[0] + 1
    assert abs(float(lses[b]) - 1 - np.log(3)) <= 2 * float(np.spacing(np.float32(2)))
    same(select(dev, x, scores, beams, flags, lse=lses))


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("beams,vocab,small", [(1, 400, 2.0 ** -20), (6, 9000, 2.0 ** -20), (6, 9000, 2.0 ** -14), (32, 20001, 2.0 ** -12)])
def test_logits_around_zero(dev, dtype, beams, vocab, small):  # noqa: F811
    """A token far above the rest, whose logits are near zero with either sign, zeros of either sign and the smallest
    floats of the type among them: what is left of them behind 200 is rounded to a step of 2^-16."""
    log("case logits around zero %s beams %d vocab %d" % (dtype, beams, vocab))
    rng = np.random.default_rng(vocab + beams)
    rows = 3 * beams
    x = small * rng.standard_normal((rows, vocab))
    x = np.where(rng.random((rows, vocab)) < 0.2, np.where(rng.random((rows, vocab)) < 0.5, 0.0, -0.0), x)
    t = torch.as_tensor(x.astype(np.float32)).to(TYPES[dtype])
    t[:, vocab // 2] = 200.0
    scores = np.full(rows, -np.inf, np.float32)
    scores[::beams] = [-1.0, -300.0, 0.0]
    same(select(dev, t, scores, beams))


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("beams,vocab", [(1, 5), (4, 700), (8, 20001)])
def test_masks_of_the_lowest_value(dev, dtype, beams, vocab):  # noqa: F811
    """Forbidden tokens at the type's lowest finite value instead of -inf: candidates like others, behind all the rest."""
    log("case lowest values %s beams %d vocab %d" % (dtype, beams, vocab))
    rng = np.random.default_rng(vocab)
    rows = 4 * beams
    t = torch.full((rows, vocab), torch.finfo(TYPES[dtype]).min, dtype=TYPES[dtype])
    t[torch.arange(rows), torch.as_tensor(rng.integers(0, vocab, rows))] = 3.0
    scores = np.full(rows, -np.inf, np.float32)
    for g in range(4):
        scores[g * beams: g * beams + max(1, beams // 4 * g)] = -2.0 - 0.5 * np.arange(max(1, beams // 4 * g))
    same(select(dev, t, scores, beams))
