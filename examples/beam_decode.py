"""Beam search under the grammar of the tags, over a paged cache that the beams of a prompt share.

    python examples/beam_decode.py

A one-layer model of random weights stands in for the language model; everything around it is the library's: the
prompts' keys and values go into the cache (kv_write), their tokens attend to them (tree_attention, a chain), and then
every step takes the newest token of each beam: decode_step advances its grammar state and forbids what may not follow,
beam_select chooses the best continuations of every prompt's beams, beam_reorder puts the states, the histories and the
mask rows into the new order.  No keys or values are copied when beams change places: all nodes of the search so far
stay in the cache, and a beam's mask row has a bit for each node on its path.
"""
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2608_24658_amd import parason as PX  # noqa: E402


class Model:
    """Random weights: token -> query, key and value heads -> attention -> logits."""

    def __init__(self, vocab, q_heads=8, heads=2, dim=64, hidden=128, device="cuda:0", seed=0):
        gen = torch.Generator(device=device).manual_seed(seed)
        r = lambda *s, f=1.0: f * torch.randn(*s, generator=gen, device=device)  # noqa: E731
        self.vocab, self.q_heads, self.heads, self.dim = vocab, q_heads, heads, dim
        self.embed = r(vocab, hidden)
        self.wq, self.wk, self.wv = (r(hidden, n * dim, f=hidden ** -0.5) for n in (q_heads, heads, heads))
        self.wo = r(q_heads * dim, vocab, f=2.0 * (q_heads * dim) ** -0.5)

    def heads_of(self, tokens):
        """Queries, keys and values of the tokens, bfloat16."""
        x = self.embed[tokens.long().clamp_min(0)]
        return tuple((x @ w).to(torch.bfloat16).view(tokens.numel(), -1, self.dim) for w in (self.wq, self.wk, self.wv))

    def logits(self, attended):
        return attended.float().flatten(1) @ self.wo


def beam_decode(model, px, prompts, beams, steps, eos_id, page=16, cache_dtype=torch.bfloat16):
    """The `beams` best streams of up to `steps` tokens behind every prompt (lists of token ids): dict of score
    [prompts * beams], history [prompts * beams, steps] (-1 behind the end of sequence) and states."""
    dev, n = model.embed.device, len(prompts)
    rows = n * beams
    i32 = lambda a: torch.tensor(a, dtype=torch.int32, device=dev)  # noqa: E731
    lens = [len(p) for p in prompts]
    # a prompt's pages hold it and every node of its search
    need = [-(-(m + beams * steps) // page) for m in lens]
    cache = PX.kv_alloc(sum(need), page, model.heads, model.dim, cache_dtype, dev)
    table = torch.full((n, max(need)), -1, dtype=torch.int32)
    for i, m in enumerate(need):
        table[i, :m] = torch.arange(m) + sum(need[:i])
    table = table.to(dev)

    # the prompts: a chain each
    tokens = i32([t for p in prompts for t in p])
    ends = torch.tensor(lens).cumsum(0)
    q, k, v = model.heads_of(tokens)
    here = PX.KVRows((ends - torch.tensor(lens)).to(dev), i32(lens), i32(lens), table, max(lens), max(lens))
    PX.kv_write(k, v, cache, here)
    first = PX.tree_attention(q, cache, here)[(ends - 1).to(dev)]
    logits = model.logits(first).repeat_interleave(beams, 0)

    # each prompt's first beam alone counts
    scores = torch.full((n, beams), float("-inf"), device=dev)
    scores[:, 0] = 0.0
    scores = scores.view(-1)
    states = PX.decode_init(rows, dev)
    px.decode_step(states, logits, None, eos_id)
    history = torch.full((rows, steps), -1, dtype=torch.int32, device=dev)
    mask = torch.zeros(rows, -(-beams * steps // 64), dtype=torch.int64, device=dev)
    starts = torch.arange(n, device=dev) * beams
    width = torch.full((n,), beams, dtype=torch.int32, device=dev)
    base, slot = i32(lens), torch.arange(rows, device=dev)
    for t in range(steps):
        new = PX.beam_select(logits, scores, beams, states=states)
        scores, tokens = new["score"], new["token"]
        states, history, mask = PX.beam_reorder(new["parent"], [states, history, mask])
        history[:, t] = tokens
        if t + 1 == steps:
            px.decode_step(states, logits, tokens, eos_id)
            break
        # the new nodes: beams * t .. of each tree, each seen by its own beam from now on
        node = slot % beams + beams * t
        mask[slot, node // 64] |= torch.ones_like(node) << (node % 64)
        nodes = width * (t + 1)
        here = PX.KVRows(starts, width, base + nodes, table, beams, max(lens) + beams * (t + 1))
        q, k, v = model.heads_of(tokens)
        PX.kv_write(k, v, cache, here)
        logits = model.logits(PX.tree_attention(q, cache, here, mask=mask, tree_lens=nodes))
        px.decode_step(states, logits, tokens, eos_id)
    return dict(score=scores, history=history, states=states)


def main():
    vocab, eos = 4096, 12
    model, px = Model(vocab), PX.Parason(list(range(12)))
    gen = torch.Generator().manual_seed(0)
    prompts = [torch.randint(13, vocab, (m,), generator=gen).tolist() for m in (40, 7, 123)]
    for dtype in (torch.bfloat16, torch.float8_e4m3fn):
        out = beam_decode(model, px, prompts, 4, 24, eos, cache_dtype=dtype)
        print(dtype, out["score"].view(len(prompts), 4).tolist())
        print(out["history"][::4].tolist())


if __name__ == "__main__":
    main()
