"""Operators of a serving and training step around the paged cache: its tables, the norm and rotation of queries and
keys, a cache held in 4 bits, and the attention that reads it.

A case is a dict of plain values.  Four kinds:

tables  kv_shrink and kv_extend: every row gives back the positions behind its last accepted one and takes room for its
        new tokens; pages come from and go to a pool on the GPU; where each new token belongs
rotate  qk_norm_rotate, or with back its backward pass qk_norm_rotate_grad: each query and key head divided by its root
        mean square, weighted, and rotated by its token's position
keep    kv_write and kv_read of a 4-bit cache: new tokens' keys and values quantised into it, and positions of it read
        back
attend  tree_attention over a 4-bit cache: "chain": each token sees all up to itself (single tokens, prompts);
        "draft": a tree of draft tokens; "threads": the threads of a <Parallel> region, every one a chain behind the
        shared prefix; "beams": the newest nodes of the tree of all beams so far

A 4-bit value is a sign, two exponent bits and a fraction bit (0, 0.5, 1, 1.5, 2, 3, 4, 6); each 32 values of a head
share a power of two, held as its exponent + 127.

With `own` false the same is computed by elementary torch operations in 32 bits (angles and the sums over all tokens in
64).
"""
import math

import numpy as np
import torch

own = False

DEVICE = "cuda:0"
TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
BYTES = {"bf16": 2, "fp16": 2, "fp32": 4}
GRID = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]
EPS = 1e-6
MAX_LEN = 1 << 30  # positions of a row
BAD_ROW, NO_PAGES = 1, 4  # bits of a row's status


def tables(name, rows, mean, new, back=0, page=16, spread="uniform", spare=0, short=False):
    return dict(name=name, kind="tables", rows=rows, mean=mean, new=new, back=back, page=page, spread=spread, spare=spare, short=short)


def rotate(name, tokens, q_heads=32, heads=8, dim=128, turned=128, given="bf16", pairs="halves", back=False, far=50300):
    return dict(name=name, kind="rotate", tokens=tokens, q_heads=q_heads, heads=heads, dim=dim, turned=turned, given=given, pairs=pairs,
                back=back, far=far)


def keep(name, rows, mean, new, read, heads=8, dim=128, page=16, given="bf16", spread="uniform"):
    return dict(name=name, kind="keep", rows=rows, mean=mean, spread=spread, new=new, read=read, heads=heads, dim=dim, page=page, given=given)


def attend(name, rows, mean, new, shape, q_heads=32, heads=8, dim=128, page=16, given="bf16", spread="uniform", nodes=0):
    return dict(name=name, kind="attend", rows=rows, mean=mean, spread=spread, new=new, shape=shape, nodes=nodes, q_heads=q_heads, heads=heads,
                dim=dim, page=page, given=given)


def listed():
    return [
        # a decode step of a serving batch of 64 rollouts: most need no page
        tables("tables_step", 64, 3500, 1),
        # finished rollouts leave, and the prompts of the next training step are admitted, in a token array of a fixed size
        tables("tables_prompts", 1024, 0, 3500, back=7000, page=64, spread="log", spare=6000),
        # one new token each of 64 rollouts
        rotate("rotate_step", 64),
        # a batch of prompts read at once, a quarter of each head not rotated
        rotate("rotate_prompts", 28001, q_heads=28, heads=4, dim=128, turned=96, given="fp16", pairs="neighbours"),
        # a small training step in float32
        rotate("rotate_train_small", 4999, q_heads=12, heads=2, dim=80, turned=32, given="fp32", back=True, far=16000),
        # the micro batch of a training step
        rotate("rotate_train", 32768, back=True),
        # one decode step of a serving batch: a token of each of 64 rollouts
        keep("keep_token", 64, 3500, 1, "new"),
        # rollouts of all lengths whose contexts are read back whole, to be handed to workers elsewhere
        keep("keep_recall", 48, 12000, 5, "all", page=24, spread="log"),
        # one token each of a few rollouts
        attend("attend_token", 16, 3500, 1, "chain"),
        # one token each of a large serving batch
        attend("attend_step", 128, 8000, 1, "chain"),
        # the draft trees of a serving batch, of all lengths
        attend("attend_draft", 48, 12000, 26, "draft", q_heads=28, heads=4, page=24, given="fp16", spread="log"),
        # a prompt
        attend("attend_prompt", 1, 0, 8192, "chain", page=64),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """A case of the listed ones' ranges that needs no more than the largest of them."""
    most = [max(work(c)[k] for c in listed()) for k in ("bytes", "flops")]
    while True:
        case = _draw(rng)
        if all(work(case)[k] <= m for k, m in zip(("bytes", "flops"), most)):
            return case


def _draw(rng):
    kind = rng.choice(["tables", "rotate", "rotate", "keep", "attend", "attend", "attend"])
    pages = [8, 16, 24, 32, 64, 100, 128, 256]
    if kind == "tables":
        rows = _log(rng, 1, 20000)
        mean = rng.choice([0, 1]) * _log(rng, 10, 12000)
        new = rng.choice([1, rng.randint(2, 80), _log(rng, 50, 12000)])
        c = dict(kind=kind, rows=rows, mean=mean, new=new, back=rng.choice([0, rng.randint(1, 200)]), page=rng.choice([1] + pages),
                 spread=rng.choice(["uniform", "log"]), spare=rng.choice([0, _log(rng, 1, 5000)]), short=rng.random() < 0.25)
        span = 3 * (mean + new) + c["back"]  # neither tables nor tokens beyond a few hundred MB
        c["rows"] = max(1, min(rows, int(6e6 / new), int(2e7 * c["page"] / span)))
        return c
    if kind == "rotate":
        q_heads, heads = rng.choice([(32, 8), (28, 4), (16, 1), (16, 16), (40, 8), (12, 2), (64, 8), (5, 5)])
        dim = rng.choice([16, 64, 80, 96, 112, 128, 128, 192, 256])
        given = rng.choice(["bf16", "bf16", "fp16", "fp32"])
        most = int(1.8e8 / ((q_heads + heads) * dim))
        return dict(kind=kind, tokens=_log(rng, 1, most), q_heads=q_heads, heads=heads, dim=dim, turned=rng.choice([dim, dim, dim // 32 * 16]),
                    given=given, pairs=rng.choice(["halves", "halves", "neighbours"]), back=rng.random() < 0.5, far=_log(rng, 10, 4000000))
    c = dict(kind=kind, spread=rng.choice(["uniform", "log"]), page=rng.choice(pages), given=rng.choice(["bf16", "bf16", "fp16"]))
    if kind == "keep":
        if rng.random() < 0.2:
            c["given"] = "fp32"
        c.update(heads=rng.choice([1, 2, 4, 8, 16]), dim=rng.choice([32, 64, 96, 128, 192, 256]))
        token = c["heads"] * c["dim"]
        c.update(mean=rng.choice([0, 1]) * _log(rng, 50, 30000), new=rng.choice([1, _log(rng, 2, 4096)]), read=rng.choice(["new", "all"]))
        c["rows"] = _log(rng, 1, max(1, min(256, int(3e8 / (token * (3 * c["mean"] + c["new"]))))))
        return c
    q_heads, heads = rng.choice([(32, 8), (28, 4), (16, 1), (16, 16), (40, 8), (12, 2), (64, 8)])
    c.update(q_heads=q_heads, heads=heads, dim=rng.choice([64, 96, 128, 128, 256]), nodes=0)
    c["shape"] = rng.choice(["chain", "chain", "draft", "threads", "beams"])
    if c["shape"] == "chain":
        c["new"] = rng.choice([1, 1, rng.randint(2, 16), _log(rng, 17, 4096)])
    elif c["shape"] == "threads":
        c["new"] = _log(rng, 100, 2500)
    elif c["shape"] == "draft":
        c["new"] = rng.randint(2, 80)
    else:
        c["new"] = rng.choice([2, 4, 5, 8, 16])
        c["nodes"] = c["new"] * _log(rng, 2, 100)
    c["mean"] = 0 if c["shape"] == "chain" and c["new"] > 16 and rng.random() < 0.5 else _log(rng, 100, 30000)
    span = (3 if c["spread"] == "log" else 1.5) * c["mean"] + c["new"] + c["nodes"]
    most = min(128, int(1.5e9 / (span * heads * c["dim"])), int(2.2e9 / (span * q_heads * c["new"])))
    if most < 1:  # one long row of many tokens: shorter
        c["mean"] = int(c["mean"] * 0.3)
        most = 1
    c["rows"] = _log(rng, 1, most)
    return c


# ---- inputs --------------------------------------------------------------------------------------------------------


def _lengths(case, mean, rng):
    """The rows' lengths around a mean, in an order of the seed's: the sizes are the case's own."""
    n, fixed = case["rows"], np.random.default_rng(0)
    if mean <= 1 or n == 1:
        return np.full(n, mean, np.int64)
    if case["spread"] == "log":  # P(L) ~ 1 / L up to three times the mean
        out = np.exp(fixed.uniform(0, math.log(3 * mean), n)).astype(np.int64)
    else:
        out = fixed.integers(max(1, mean // 2), mean + mean // 2 + 1, n)
    return rng.permutation(out)


def _ints(a, dtype):
    return torch.as_tensor(np.ascontiguousarray(a)).to(device=DEVICE, dtype=dtype)


def _page_table(need, total, rng):
    """[rows, most] page numbers in no order, -1 behind each row's own; and the pages that belong to nobody."""
    order = rng.permutation(total)
    pages = np.full((len(need), max(1, int(need.max()))), -1, np.int32)
    pages[np.arange(pages.shape[1])[None, :] < need[:, None]] = order[: int(need.sum())]
    return pages, order[int(need.sum()):]


def _sizes_of_tables(case, rng):
    """Positions that are kept, that are held before the step, and new ones, of every row."""
    kept = _lengths(case, case["mean"], rng)
    new = _lengths(case, case["new"], rng)
    if case["new"] > 1:
        new[np.argsort(new, kind="stable")[10::20]] = 0  # a row in twenty waits
    back = np.random.default_rng(1).integers(0, case["back"] + 1, case["rows"])
    return kept, kept + back, new


def _prepare_tables(case, seed):
    rng = np.random.default_rng(seed)
    page = case["page"]
    kept, held, new = _sizes_of_tables(case, rng)
    # as many pages and entries as any pairing of the lengths needs
    total = int(sum((-(-n // page)).sum() for n in (kept, held - kept, new))) + 7
    table, free = _page_table(-(-held // page), total, rng)
    pages = np.full((case["rows"], -(-int(kept.max() + (held - kept).max() + new.max()) // page)), -1, np.int32)
    pages[:, : table.shape[1]] = table
    if case["short"]:  # the pool ends before the last rows are served
        before, between, after = ((-(-n // page)).sum() for n in (held, kept, kept + new))
        free = free[: max(0, int((after - between) // 2 - (before - between)))]
    stack = np.full(total, -1, np.int32)
    stack[: free.size] = free
    return dict(free=_ints(stack, torch.int32), count=_ints([free.size], torch.int32), kept=_ints(kept, torch.int32),
                held=_ints(held, torch.int32), pages=_ints(pages, torch.int32), new=_ints(new, torch.int32), page=page,
                total=int(new.sum()) + case["spare"])


def _prepare_rotate(case, seed):
    gen = torch.Generator(device=DEVICE).manual_seed(seed)
    n, q_heads, heads, dim, given = case["tokens"], case["q_heads"], case["heads"], case["dim"], TYPES[case["given"]]
    # queries, keys and values as one projection leaves them; some channels are larger than others
    size = torch.exp(0.7 * torch.randn(q_heads + 2 * heads, dim, generator=gen, device=DEVICE))
    x = (torch.randn(n, q_heads + 2 * heads, dim, generator=gen, device=DEVICE) * size).to(given)
    at = torch.randint(0, case["far"], (n,), generator=gen, device=DEVICE, dtype=torch.int32)
    if not case["back"]:  # a token in thirty is padding
        at = torch.where(torch.rand(n, generator=gen, device=DEVICE) < 1 / 30, -1, at)
    turned = case["turned"]
    freqs = torch.pow(1e6, -torch.arange(0, turned, 2, device=DEVICE, dtype=torch.float64) / max(1, turned))
    st = dict(q=x[:, :q_heads], k=x[:, q_heads: q_heads + heads], at=at, freqs=freqs, pairs=case["pairs"])
    st["q_weight"], st["k_weight"] = (1 + 0.3 * torch.randn(2, dim, generator=gen, device=DEVICE)).to(given)
    if case["back"]:
        g = (1e-3 * torch.randn(n, q_heads + heads, dim, generator=gen, device=DEVICE)).to(given)
        st["dq"], st["dk"] = g[:, :q_heads], g[:, q_heads:]
    return st


def _pool(case, positions, rng, gen):
    """A pool of pages, a table that gives every row its pages in no order, and the pool's contents."""
    page, heads, dim = case["page"], case["heads"], case["dim"]
    need = -(-positions // page)
    total = int(need.sum()) + 3  # pages that belong to nobody
    pages, _ = _page_table(need, total, rng)
    # keys and values lie head by head within a page; the views are [pages, page, heads, ...]
    size = (2, total, heads, page, dim // 2)
    codes = torch.randint(0, 256, size, generator=gen, device=DEVICE, dtype=torch.uint8)
    scales = torch.randint(125, 127, size[:-1] + (dim // 32,), generator=gen, device=DEVICE, dtype=torch.uint8)
    return dict(pages=_ints(pages, torch.int32), cache=[c.view(torch.float4_e2m1fn_x2).permute(0, 2, 1, 3) for c in codes],
                scales=[s.view(torch.float8_e8m0fnu).permute(0, 2, 1, 3) for s in scales])


def _rows(new, positions, pages):
    """What describes the rows of a call: where their new tokens are, how many, how many positions the cache holds with
    them, their pages, and the largest of both."""
    starts = np.cumsum(new) - new
    return (_ints(starts, torch.int64), _ints(new, torch.int32), _ints(positions, torch.int32), pages, int(new.max()), int(positions.max()))


def _words(seen):
    """Truth values [rows, n] as 64-bit words [rows, ceil(n / 64)], the first one in the lowest bit."""
    rows, n = seen.shape
    bits = np.zeros((rows, -(-n // 64) * 64), np.uint8)
    bits[:, :n] = seen
    return np.packbits(bits, axis=1, bitorder="little").view(np.int64)


def _prepare_keep(case, seed):
    rng, gen = np.random.default_rng(seed), torch.Generator(device=DEVICE).manual_seed(seed)
    new = _lengths(case, case["new"], rng)
    positions = _lengths(case, case["mean"], rng) + new
    st = _pool(case, positions, rng, gen)
    size = torch.exp(0.7 * torch.randn(2, 1, case["heads"], case["dim"], generator=gen, device=DEVICE))
    x = torch.randn(2, int(new.sum()), case["heads"], case["dim"], generator=gen, device=DEVICE) * size
    st["k"], st["v"] = x.to(TYPES[case["given"]])
    read = new if case["read"] == "new" else positions
    return dict(st, write=_rows(new, positions, st["pages"]), read=_rows(read, positions, st["pages"]), total=int(read.sum()))


def _parents(case, n, rng):
    """Parents of a tree's nodes (-1: none), every one before its children."""
    i = np.arange(n)
    if case["shape"] == "threads":  # two to eight chains
        cuts = np.sort(rng.choice(np.arange(1, n), size=min(n - 1, int(rng.integers(1, 8))), replace=False)) if n > 1 else i[:0]
        return np.where(np.isin(i, cuts) | (i == 0), -1, i - 1)
    if case["shape"] == "beams":  # every step's nodes choose among the step before
        w = case["new"]
        return np.where(i < w, -1, (i // w - 1) * w + rng.integers(0, w, n))
    # the first tokens a choice of their own, later ones behind one of the last eight
    return np.where(i < 2, -1, i - rng.integers(1, np.clip(i, 1, 8) + 1))


def _seen(parents):
    """[n, n]: node i sees itself and its ancestors."""
    n = len(parents)
    seen = np.zeros((n, n), bool)
    for i in range(n):
        if parents[i] >= 0:
            seen[i] = seen[parents[i]]
        seen[i, i] = True
    return seen


def _prepare_attend(case, seed):
    rng, gen = np.random.default_rng(seed), torch.Generator(device=DEVICE).manual_seed(seed)
    q_heads, dim, shape = case["q_heads"], case["dim"], case["shape"]
    n = np.full(case["rows"], case["new"], np.int64) if case["new"] <= 80 else _lengths(case, case["new"], rng)
    nodes = np.full(case["rows"], case["nodes"], np.int64) if shape == "beams" else n
    positions = _lengths(case, case["mean"], rng) + nodes
    st = _pool(case, positions, rng, gen)
    st["q"] = torch.randn(int(n.sum()), q_heads, dim, generator=gen, device=DEVICE).to(TYPES[case["given"]])
    st.update(rows=_rows(n, positions, st["pages"]), mask=None, tree=None, scale=dim ** -0.5)
    if shape != "chain":
        words = -(-int(nodes.max()) // 64)
        made = [_words(_seen(_parents(case, int(t), rng))[-int(m):]) for t, m in zip(nodes, n)]
        mask = np.concatenate([np.pad(m, ((0, 0), (0, words - m.shape[1]))) for m in made])
        st.update(mask=_ints(mask, torch.int64), tree=_ints(nodes, torch.int32))
    return st


def prepare(case, seed):
    st = dict(tables=_prepare_tables, rotate=_prepare_rotate, keep=_prepare_keep, attend=_prepare_attend)[case["kind"]](case, seed)
    return dict(st, kind=case["kind"])


# ---- one pass ------------------------------------------------------------------------------------------------------


def run(st):
    kind = st["kind"]
    if own:
        from paper_2608_24658_amd import parason as PX

        if kind == "tables":
            pool = PX.KVPool(st["free"], st["count"])
            PX.kv_shrink(pool, st["kept"], st["held"], st["pages"], st["page"])
            step = PX.kv_extend(pool, st["new"], st["held"], st["pages"], st["page"], st["total"])
            return dict(step, kv_lens=st["held"], pages=st["pages"], free=st["free"], count=st["count"])
        if kind == "rotate":
            more = dict(q_weight=st["q_weight"], k_weight=st["k_weight"], eps=EPS, interleaved=st["pairs"] == "neighbours")
            if "dq" in st:
                return PX.qk_norm_rotate_grad(st["dq"], st["dk"], st["q"], st["k"], st["at"], st["freqs"], **more)
            q, k = PX.qk_norm_rotate(st["q"], st["k"], st["at"], st["freqs"], **more)
            return dict(q=q, k=k)
        kept = PX.KVCache(*st["cache"], *st["scales"])
        if kind == "attend":
            out, lse = PX.tree_attention(st["q"], kept, PX.KVRows(*st["rows"]), mask=st["mask"], tree_lens=st["tree"], scale=st["scale"],
                                         lse=True)
            return dict(out=out, lse=lse)
        PX.kv_write(st["k"], st["v"], kept, PX.KVRows(*st["write"]))
        k, v = PX.kv_read(kept, PX.KVRows(*st["read"]), st["total"], st["k"].dtype)
        return dict(k=k, v=v)
    if kind == "tables":
        _plain_shrink(st)
        return _plain_extend(st)
    if kind == "rotate":
        return _plain_rotate_grad(st) if "dq" in st else _plain_rotate(st)
    return dict(keep=_plain_keep, attend=_plain_attend)[kind](st)


def _pages_of(n, page):
    return (n + (page - 1)) // page


def _plain_shrink(st):
    """The pages behind each row's last kept position go onto the pool, the first row's first page last."""
    held, kept, pages, page = st["held"].long(), st["kept"].long(), st["pages"], st["page"]
    kept = torch.where((kept >= 0) & (kept <= held), kept, held)
    had, keeps = _pages_of(held, page), _pages_of(kept, page)
    freed = had - keeps
    before = torch.cumsum(freed, 0) - freed
    col = torch.arange(pages.shape[1], device=DEVICE)
    gone = (col >= keeps[:, None]) & (col < had[:, None])
    to = st["count"].long() + freed.sum() - 1 - (before[:, None] + col - keeps[:, None])
    # what stays in the table goes to a place behind the pool
    stack = torch.cat([st["free"], st["free"][:1]])
    stack[torch.where(gone, to, st["free"].numel()).reshape(-1)] = pages.reshape(-1)
    st["free"].copy_(stack[:-1])
    st["count"] += freed.sum().int()
    pages.masked_fill_(gone, -1)
    st["held"].copy_(kept)


def _plain_extend(st):
    held, new, pages, page, total = st["held"].long(), st["new"].long(), st["pages"], st["page"], st["total"]
    given = new.clamp_min(0)
    ends = torch.cumsum(given, 0)
    starts = ends - given
    after = held + given
    good = (new >= 0) & (held >= 0) & (after <= min(pages.shape[1] * page, MAX_LEN)) & (ends <= total)
    had = _pages_of(held, page)
    need = torch.where(good, _pages_of(after, page) - had, 0)
    upto = torch.cumsum(need, 0)
    served = good & ((need == 0) | (upto <= st["count"]))
    need = torch.where(served, need, 0)
    col = torch.arange(pages.shape[1], device=DEVICE)
    fresh = (col >= had[:, None]) & (col < (had + need)[:, None])
    at = st["count"].long() - 1 - ((upto - need)[:, None] + col - had[:, None])
    pages.copy_(torch.where(fresh, st["free"][torch.where(fresh, at, 0)], pages))
    st["count"] -= need.sum().int()
    # the tokens: whose, which position, which slot
    t = torch.arange(total, device=DEVICE)
    row = torch.searchsorted(ends, t, right=True)
    there = row < ends.numel()
    row = torch.where(there, row, 0)
    there &= served[row]
    where = held[row] + t - starts[row]
    slot = pages[row, torch.where(there, where // page, 0)].long() * page + where % page
    st["held"].copy_(torch.where(served, after, held))
    status = torch.where(good, torch.where(served, 0, NO_PAGES), BAD_ROW)
    return dict(lengths=torch.where(served, new, 0).int(), starts=starts.clamp_max(total), positions=torch.where(there, where, -1).int(),
                slots=torch.where(there, slot, -1), rows=torch.where(there, row, -1).int(), status=status.int(), kv_lens=st["held"],
                pages=pages, free=st["free"], count=st["count"])


def _turns(st):
    """Cosines and sines [tokens, 1, pairs] of every token's angles."""
    angle = st["at"].double()[:, None, None] * st["freqs"]
    return torch.cos(angle).float(), torch.sin(angle).float()


def _split(x, st):
    """The two halves of the rotated values' pairs, and the values that are not rotated."""
    n = 2 * st["freqs"].numel()
    if st["pairs"] == "halves":
        return x[..., : n // 2], x[..., n // 2: n], x[..., n:]
    return x[..., 0:n:2], x[..., 1:n:2], x[..., n:]


def _joined(a, b, rest, st):
    turned = torch.cat([a, b], -1) if st["pairs"] == "halves" else torch.stack([a, b], -1).flatten(-2)
    return torch.cat([turned, rest], -1)


def _plain_rotate(st):
    cos, sin = _turns(st)

    def one(x, weight):
        y = x.float()
        y = y * torch.rsqrt((y * y).mean(-1, keepdim=True) + EPS) * weight.float()
        a, b, rest = _split(y, st)
        y = _joined(a * cos - b * sin, b * cos + a * sin, rest, st)
        return torch.where((st["at"] >= 0)[:, None, None], y, 0.0).to(x.dtype)

    return dict(q=one(st["q"], st["q_weight"]), k=one(st["k"], st["k_weight"]))


def _plain_rotate_grad(st):
    cos, sin = _turns(st)

    def one(x, g, weight):
        y, there = x.float(), (st["at"] >= 0)[:, None, None]
        a, b, rest = _split(torch.where(there, g.float(), 0.0), st)
        g = _joined(a * cos + b * sin, b * cos - a * sin, rest, st)
        r = torch.rsqrt((y * y).mean(-1, keepdim=True) + EPS)
        y = y * r
        dw = torch.where(there, g * y, 0.0).sum((0, 1), dtype=torch.float64)
        g = g * weight.float()
        dx = torch.where(there, r * (g - y * (g * y).mean(-1, keepdim=True)), 0.0)
        return dx.to(x.dtype), dw.float()

    (q, q_weight), (k, k_weight) = one(st["q"], st["dq"], st["q_weight"]), one(st["k"], st["dk"], st["k_weight"])
    return dict(q=q, k=k, q_weight=q_weight, k_weight=k_weight)


def _places(rows, n, page):
    """Page and slot of the n tokens that a call's rows name."""
    starts, lengths, positions, pages, _, _ = rows
    row = torch.repeat_interleave(torch.arange(starts.numel(), device=DEVICE), lengths.long(), output_size=n)
    at = positions.long()[row] - lengths.long()[row] + torch.arange(n, device=DEVICE) - starts[row]
    return pages[row, at // page].long(), at % page


def _store(x, cache, scale, page, slot):
    x = x.float().unflatten(-1, (-1, 32))
    top = x.abs().amax(-1)
    fine = torch.isfinite(top)
    # the least power of two for which the largest value is at most 7 times it
    part, e = torch.frexp(torch.where(fine, top, 0.0))
    e = (e - 3 + (part > 0.875)).clamp(-120, 125)
    y = x * ((127 - e) << 23).view(torch.float32)[..., None]
    a = y.abs()
    code = (a > 0.25).int() + (a >= 0.75) + (a > 1.25) + (a >= 1.75) + (a > 2.5) + (a >= 3.5) + (a > 5) + 8 * torch.signbit(y)
    code = torch.where(fine[..., None], code, 0).flatten(-2)
    cache.view(torch.uint8)[page, slot] = (code[..., 0::2] + 16 * code[..., 1::2]).to(torch.uint8)
    scale.view(torch.uint8)[page, slot] = torch.where(fine, e + 127, 255).to(torch.uint8)


def _load(cache, scale, page, slot):
    x, e = cache.view(torch.uint8)[page, slot].int(), scale.view(torch.uint8)[page, slot].int()
    code = torch.stack([x & 15, x >> 4], -1).flatten(-2)
    y = torch.tensor(GRID + [-v for v in GRID], device=DEVICE)[code].unflatten(-1, (-1, 32))
    return (y * torch.where(e == 255, float("nan"), (e << 23).view(torch.float32))[..., None]).flatten(-2)


def _plain_keep(st):
    page = st["cache"][0].shape[1]
    at = _places(st["write"], st["k"].shape[0], page)
    _store(st["k"], st["cache"][0], st["scales"][0], *at)
    _store(st["v"], st["cache"][1], st["scales"][1], *at)
    at = _places(st["read"], st["total"], page)
    given = st["k"].dtype
    return dict(k=_load(st["cache"][0], st["scales"][0], *at).to(given), v=_load(st["cache"][1], st["scales"][1], *at).to(given))


def _plain_attend(st):
    """All rows at once, padded to the longest."""
    q, scales, mask = st["q"], st["scales"], st["mask"]
    starts, lengths, positions, pages, n, kv = st["rows"]
    k, v = st["cache"]
    page, heads = k.shape[1:3]
    rows, q_heads, dim = starts.numel(), q.shape[1], q.shape[2]
    # keys and values [rows, heads, kv, dim], zero behind a row's end
    at = torch.arange(kv, device=DEVICE)
    there = at[None, :] < positions[:, None]
    pg, slot = torch.where(there, pages[:, at // page], 0).long(), (at % page).expand(rows, kv)
    keys = torch.where(there[..., None, None], _load(k, scales[0], pg, slot), 0.0).permute(0, 2, 3, 1)
    values = torch.where(there[..., None, None], _load(v, scales[1], pg, slot), 0.0).permute(0, 2, 1, 3)
    # queries [rows, heads, group * n, dim]; a row's tokens beyond its own are its last one again
    token = torch.arange(n, device=DEVICE)
    which = starts[:, None] + torch.minimum(token[None, :], lengths[:, None].long() - 1)
    x = q[which].float().reshape(rows, n, heads, q_heads // heads, dim).permute(0, 2, 3, 1, 4).reshape(rows, heads, -1, dim)
    if mask is None:
        seen = at[None, None, :] <= (positions - lengths)[:, None, None] + token[None, :, None]
    else:
        bit = at[None, :] - (positions - st["tree"])[:, None]
        word = (bit >> 6).clamp(0, mask.shape[1] - 1)[:, None, :].expand(rows, n, kv)
        seen = (torch.gather(mask[which], 2, word) >> (bit & 63)[:, None, :]) & 1 != 0
        seen = (seen | (bit < 0)[:, None, :]) & there[:, None, :]
    score = torch.matmul(x, keys).reshape(rows, heads, -1, n, kv) * st["scale"]
    score = torch.where(seen[:, None, None], score, float("-inf"))
    top = score.amax(-1, keepdim=True).clamp_min(-3e38)
    p = torch.exp(score - top)
    total = p.sum(-1, keepdim=True)
    lse = (top + torch.log(total)).reshape(rows, q_heads, n).permute(0, 2, 1)
    p = (p / torch.where(total > 0, total, 1.0)).reshape(rows, heads, -1, kv)
    out = torch.matmul(p, values).reshape(rows, q_heads, n, dim).permute(0, 2, 1, 3)
    mine = token[None, :] < lengths[:, None]
    return dict(out=out[mine].to(q.dtype), lse=lse[mine])


# ---- what a pass cannot do without ---------------------------------------------------------------------------------


def _total(case, mean):
    return int(_lengths(case, mean, np.random.default_rng(0)).sum())


def work(case):
    kind = case["kind"]
    if kind == "tables":
        # lengths read and written, the pages that move, and 16 bytes for each token
        kept, held, new = _sizes_of_tables(case, np.random.default_rng(0))
        before, between, after = (-(-n // case["page"]) for n in (held, kept, kept + new))
        moved = int((before - between + after - between).sum())
        return dict(bytes=case["rows"] * 32 + moved * 12 + 16 * (int(new.sum()) + case["spare"]), flops=0)
    if kind == "rotate":
        values = case["tokens"] * (case["q_heads"] + case["heads"]) * case["dim"]
        return dict(bytes=values * BYTES[case["given"]] * (3 if case["back"] else 2) + 4 * case["tokens"], flops=values * (14 if case["back"] else 7))
    heads, dim = case["heads"], case["dim"]
    slot = 2 * heads * (dim // 2 + dim // 32)
    if kind == "keep":
        new, old = _total(case, case["new"]), _total(case, case["mean"])
        read = new if case["read"] == "new" else new + old
        given = 2 * heads * dim * BYTES[case["given"]]
        return dict(bytes=new * (given + slot) + read * (given + slot), flops=2 * heads * dim * (3 * new + read))
    rows, q_heads = case["rows"], case["q_heads"]
    n = np.full(rows, case["new"], np.int64) if case["new"] <= 80 else _lengths(case, case["new"], np.random.default_rng(0))
    nodes = case["nodes"] if case["shape"] == "beams" else n
    old = _lengths(case, case["mean"], np.random.default_rng(0))
    # pairs of a query and a position that it sees: all of the prefix, and of the tree its own path
    path = dict(chain=(n + 1) / 2, threads=(n / 4 + 1) / 2, draft=1 + np.log2(n) * 2, beams=np.full(rows, case["nodes"] / case["new"]))[case["shape"]]
    pairs = float((n * (old.mean() + path)).sum())
    return dict(bytes=float((old + nodes).sum()) * slot + float(n.sum()) * q_heads * (2 * dim * BYTES[case["given"]] + 4),
                flops=4 * dim * q_heads * pairs)


# ---- the same in 64 bits -------------------------------------------------------------------------------------------


def _e2m1(x):
    """The nearest of the 16 values, ties to the one with an even fraction bit: steps of 0.5, 1 and 2 by magnitude."""
    a = x.abs()
    step = torch.where(a < 2, 0.5, torch.where(a < 4, 1.0, 2.0)).double()
    return torch.copysign((torch.round(a / step) * step).clamp_max(6.0), x)


def exact(case, seed):
    kind = case["kind"]
    if kind == "tables":
        return None
    st = prepare(case, seed)
    if kind == "rotate":
        # a pair is a complex number, the rotation a product with one of size 1
        there = (st["at"] >= 0)[:, None, None]
        angle = st["at"].double()[:, None] * st["freqs"][None]
        turn = torch.polar(torch.ones_like(angle), angle)[:, None]
        n = 2 * st["freqs"].numel()

        def rotated(x, by):
            if n == 0:
                return x
            z = x[..., :n].unflatten(-1, (2, -1)).transpose(-1, -2) if st["pairs"] == "halves" else x[..., :n].unflatten(-1, (-1, 2))
            z = torch.view_as_real(torch.view_as_complex(z.contiguous()) * by)
            z = (z.transpose(-1, -2) if st["pairs"] == "halves" else z).flatten(-2)
            return torch.cat([z, x[..., n:]], -1)

        out = {}
        for name in "qk":
            x, w = st[name].double(), st[name + "_weight"].double()
            rms = torch.sqrt(x.square().mean(-1, keepdim=True) + EPS)
            if not case["back"]:
                out[name] = rotated(x / rms * w, turn) * there
                continue
            g = rotated(st["d" + name].double(), turn.conj()) * there
            out[name + "_weight"] = (g * x / rms).sum((0, 1))
            out[name] = g * w / rms - x * (g * w * x).sum(-1, keepdim=True) / (case["dim"] * rms ** 3)
            del x, g
        return out
    cache = [c.view(torch.uint8) for c in st["cache"]]
    scales = [s.view(torch.uint8) for s in st["scales"]]
    grid = torch.tensor(GRID + [-v for v in GRID], dtype=torch.float64, device=DEVICE)

    def values(which, row, lo, hi):
        """Positions lo .. hi of a row's cached keys or values, in 64 bits."""
        at = torch.arange(lo, hi, device=DEVICE)
        pg, slot = st["pages"][row].long()[at // case["page"]], at % case["page"]
        x = cache[which][pg, slot].long()
        x = grid[torch.stack([x % 16, x // 16], -1)].flatten(-2)
        return x * torch.exp2(scales[which][pg, slot].double() - 127).repeat_interleave(32, -1)

    if kind == "keep":
        starts, lengths, positions = (t.tolist() for t in st["write"][:3])
        reads = st["read"][1].tolist()
        out = dict(k=[], v=[])
        for which, name in enumerate("kv"):
            for i in range(case["rows"]):
                x = st[name][starts[i]: starts[i] + lengths[i]].double().unflatten(-1, (-1, 32))
                s = torch.exp2(torch.ceil(torch.log2(x.abs().amax(-1, keepdim=True) / 7)).clamp(-120, 125))
                x = (_e2m1(x / s) * s).flatten(-2)
                out[name].append(torch.cat([values(which, i, positions[i] - reads[i], positions[i] - lengths[i]), x]))
            out[name] = torch.cat(out[name])
        return out
    q, scale = st["q"], st["scale"]
    starts, lengths, positions = (t.tolist() for t in st["rows"][:3])
    nodes = st["tree"].tolist() if st["tree"] is not None else lengths
    group = case["q_heads"] // case["heads"]
    if 1e-13 * 4 * case["dim"] * case["q_heads"] * sum(a * b for a, b in zip(lengths, positions)) > 1:
        return None
    out, lse = torch.empty(q.shape, dtype=torch.float64, device=DEVICE), torch.empty(q.shape[:2], dtype=torch.float64, device=DEVICE)
    for i in range(case["rows"]):
        kv, base = positions[i], positions[i] - nodes[i]
        k, v = values(0, i, 0, kv), values(1, i, 0, kv)
        for lo in range(0, lengths[i], 512):
            hi = min(lengths[i], lo + 512)
            seen = torch.ones(hi - lo, kv, dtype=torch.bool, device=DEVICE)
            if st["mask"] is None:
                seen = torch.arange(kv, device=DEVICE)[None, :] <= torch.arange(kv - lengths[i] + lo, kv - lengths[i] + hi, device=DEVICE)[:, None]
            else:
                words = st["mask"][starts[i] + lo: starts[i] + hi]
                bits = (words[:, :, None] >> torch.arange(64, device=DEVICE)) & 1
                seen[:, base:] = bits.reshape(hi - lo, -1)[:, : nodes[i]] != 0
            for h in range(case["q_heads"]):
                a = q[starts[i] + lo: starts[i] + hi, h].double() @ k[:, h // group].t() * scale
                a = a.masked_fill(~seen, float("-inf"))
                z = torch.logsumexp(a, 1)
                lse[starts[i] + lo: starts[i] + hi, h] = z
                out[starts[i] + lo: starts[i] + hi, h] = torch.exp(a - z[:, None]) @ v[:, h // group]
    return dict(out=out, lse=lse)
