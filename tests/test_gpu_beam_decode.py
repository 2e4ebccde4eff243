"""The example of constrained beam decoding: every stream it returns, gone over token by token without a cache.

The model is evaluated again in 64 bits over prompt and stream (dense causal attention, from the same bfloat16 queries,
keys and values), under the masks that decode_step gives for the stream alone; the sum of its log probabilities is the
beam's score within what rounding allows: an attended value is off by at most 2^-9 of the largest |v| for the weights
and 2^-9 of itself for its own rounding (2^-20 for everything in float32 beside them), each logit by the sum of that
over its column of weights, each log probability by twice the largest of these."""
import numpy as np
import pytest

from gpu_util import log
from paper_2608_24658_amd import parason as PX

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

EOS, VOCAB = 12, 700


@pytest.fixture(scope="module")
def dev():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    return torch.device("cuda:0")


def example():
    import importlib.util
    import os

    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "beam_decode.py")
    spec = importlib.util.spec_from_file_location("beam_decode", path)
    mod = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(mod)
    return mod


@pytest.mark.parametrize("beams,steps,page", [(1, 6, 16), (4, 20, 16), (5, 30, 8)])
def test_scores_are_the_streams_own(dev, beams, steps, page):
    log("case beam decode %d beams %d steps" % (beams, steps))
    ex = example()
    model, px = ex.Model(VOCAB, device=dev, seed=beams), PX.Parason(list(range(12)))
    rng = np.random.default_rng(beams)
    prompts = [rng.integers(13, VOCAB, m).tolist() for m in (9, 33, 1)]
    out = ex.beam_decode(model, px, prompts, beams, steps, EOS, page=page)
    score, history = out["score"].cpu().view(len(prompts), beams), out["history"].cpu().view(len(prompts), beams, steps)
    assert torch.equal(score, score.sort(1, descending=True).values)
    column = model.wo.double().abs().sum(0).max().item()
    for i, prompt in enumerate(prompts):
        seen = set()
        for b in range(beams):
            if not torch.isfinite(score[i, b]):
                continue
            h = [t for t in history[i, b].tolist() if t >= 0]
            assert history[i, b].tolist() == h + [-1] * (steps - len(h)) and (len(h) == steps or h[-1] == EOS)
            seen.add(tuple(h))
            q, k, v = (x.double().cpu() for x in model.heads_of(torch.tensor(prompt + h[:-1], device=dev)))
            group = model.q_heads // model.heads
            s = torch.stack([q[:, j] @ k[:, j // group].T for j in range(model.q_heads)]) * model.dim ** -0.5
            p = torch.softmax(s.masked_fill(torch.ones(s.shape[1:]).triu(1).bool(), float("-inf")), -1)
            a = torch.stack([p[j] @ v[:, j // group] for j in range(model.q_heads)], 1)[len(prompt) - 1:]
            logits = (a.flatten(1) @ model.wo.double().cpu()).to(dev).float()
            states, total = PX.decode_init(1, dev), 0.0
            for t, token in enumerate(h):
                row = logits[t: t + 1].clone()
                last = torch.tensor(h[t - 1: t], dtype=torch.int32, device=dev) if t else None
                px.decode_step(states, row, last, EOS)
                total += torch.log_softmax(row.double(), 1)[0, token].item()
            assert np.isfinite(total)  # no token that the grammar forbids
            each = (2.0 ** -9 + 2.0 ** -9 + 2.0 ** -20) * v.abs().max().item()
            assert abs(total - score[i, b].item()) <= len(h) * 2 * each * column + 1e-5 * abs(total), (i, b)
        assert len(seen) == int(torch.isfinite(score[i]).sum())
    flags = out["states"].view(torch.int32).view(-1, 4)[:, 3].cpu()
    assert not ((flags & 1 != 0) & torch.isfinite(out["score"].cpu())).any()


def test_example_runs(dev, capsys):
    log("case beam decode example")
    example().main()
    assert "float8" in capsys.readouterr().out


def test_a_step_in_a_graph(dev):
    """A step's write, read back, attention, choice and reordering in one graph, replayed with other work between the
    replays: every replay as the eager step."""
    log("case beam step in a graph")
    beams, heads, dim, vocab, kv = 4, 2, 64, 3000, 200
    gen = torch.Generator(device=dev).manual_seed(0)
    r = lambda *s: torch.randn(*s, generator=gen, device=dev)  # noqa: E731
    cache = PX.kv_alloc(30, 16, heads, dim, torch.float8_e4m3fn, dev)
    table = torch.arange(28, dtype=torch.int32, device=dev).view(2, 14)
    i32 = lambda a: torch.tensor(a, dtype=torch.int32, device=dev)  # noqa: E731
    two = lambda n: PX.KVRows(torch.tensor([0, n], device=dev), i32([n, n]), i32([kv, kv]), table, n, kv)  # noqa: E731
    old, new = two(kv), two(beams)
    before = r(2, 2 * kv, heads, dim)
    q, k, v = r(8, 8, dim).bfloat16(), r(8, heads, dim).bfloat16(), r(8, heads, dim).bfloat16()
    mask = torch.randint(0, 2 ** 12, (8, 1), generator=gen, device=dev) | 1
    trees, logits, scores = i32([12, 12]), r(8, vocab), -torch.rand(8, generator=gen, device=dev)
    history = torch.randint(0, vocab, (8, 77), generator=gen, device=dev, dtype=torch.int32)

    def step():
        PX.kv_write(k, v, cache, new)
        back = PX.kv_read(cache, new, 8, torch.bfloat16)
        out, lse = PX.tree_attention(q, cache, new, mask=mask, tree_lens=trees, lse=True)
        best = PX.beam_select(logits, scores, beams)
        moved = PX.beam_reorder(best["parent"], [history, mask])
        return [*back, out, lse, *best.values(), *moved]

    PX.kv_write(before[0], before[1], cache, old)
    want = [t.clone() for t in step()]
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step()
    for _ in range(3):
        PX.kv_write(before[1], before[0], cache, old)
        PX.kv_write(before[0], before[1], cache, old)
        for t in got:
            t.zero_()
        (r(1000) * 2).sum().item()
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(want, got):
            assert torch.equal(a, b)
