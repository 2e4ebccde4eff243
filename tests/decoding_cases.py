"""Caches, rows and trees for the tests of the decoding operators."""
import numpy as np

from paper_2608_24658_amd import parason as PX

KINDS = ("bf16", "fp16", "fp8", "int8")


def torch_type(kind):
    import torch

    return {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32, "fp8": torch.float8_e4m3fn,
            "int8": torch.int8}[kind]


class Paged:
    """A cache with pages in random order, the rows' page tables, and what every position holds (float32)."""

    def __init__(self, dev, kv_lens, page, heads, dim, kind, seed, layout="heads", spare=3, pad=0, extra_slots=0):
        import torch

        self.rng = np.random.default_rng(seed)
        self.kind, self.page, self.heads, self.dim = kind, page, heads, dim
        self.kv_lens = np.asarray(kv_lens, np.int64)
        need = -(-(self.kv_lens + extra_slots) // page)
        self.n_pages = int(need.sum()) + spare
        order = self.rng.permutation(self.n_pages)[: int(need.sum())]
        self.pages = np.full((len(kv_lens), max(1, int(need.max(initial=0)))), -7, np.int32)
        self.pages[np.arange(self.pages.shape[1])[None, :] < need[:, None]] = order
        dt = torch_type(kind)
        code = kind in ("fp8", "int8")
        shape = dict(heads=(self.n_pages, heads, page, dim + pad), slots=(self.n_pages, page, heads, dim + pad))[layout]
        swap = (0, 2, 1, 3) if layout == "heads" else (0, 1, 2, 3)
        # what no one has written: NaN in 16 bits, NaN scales in 8
        junk = torch.full(shape, 0x7F if code else 0x7FFF, dtype=torch.uint8 if code else torch.int16)
        self.kv = [junk.clone().to(dev).view(dt).permute(swap)[..., :dim] for _ in "kv"]
        self.scales = [torch.full(shape[:3], float("nan")).to(dev).permute(swap[:3]) for _ in "kv"] if code else []
        self.cache = PX.KVCache(*self.kv, *self.scales)
        self.dev = dev

    def place(self, row, pos):
        pos = np.asarray(pos)
        return self.pages[row, pos // self.page].astype(np.int64), pos % self.page

    def fill(self, values_of):
        """Put values_of(row, n) -> float32 [2, n, heads, dim] into the cache without the library (the oracle's codes);
        keeps the 64-bit values of what it now holds in self.held[row]."""
        import torch
        from oracle import decoding_oracle as D

        self.held = []
        host = [t.cpu().clone() for t in (x.view(torch.uint8) if self.scales else x for x in self.kv)]
        host_s = [t.cpu().clone() for t in self.scales]
        for i, n in enumerate(self.kv_lens):
            x = np.asarray(values_of(i, int(n)), np.float32)
            pg, slot = self.place(i, np.arange(int(n)))
            held = []
            for w in range(2):
                if self.scales:
                    codes, s = D.quantise(x[w], self.kind)
                    host[w][pg, slot] = torch.from_numpy(codes.view(np.uint8))
                    host_s[w][pg, slot] = torch.from_numpy(s)
                    held.append(D.values(codes, s, self.kind).astype(np.float64))
                else:
                    t = torch.from_numpy(x[w]).to(self.kv[w].dtype)
                    host[w][pg, slot] = t
                    held.append(t.double().numpy())
            self.held.append(held)
        for w in range(2):
            (self.kv[w].view(torch.uint8) if self.scales else self.kv[w]).copy_(host[w])
            if self.scales:
                self.scales[w].copy_(host_s[w])
        return self

    def rows(self, lengths, gap=0, kv_lens=None):
        """KVRows of `lengths` tokens a row, `gap` unused tokens in front of each row; and the number of tokens."""
        import torch

        lengths = np.asarray(lengths, np.int64)
        kv_lens = self.kv_lens if kv_lens is None else np.asarray(kv_lens, np.int64)
        starts = np.cumsum(lengths + gap) - lengths
        t = lambda a, dt: torch.as_tensor(np.ascontiguousarray(a)).to(device=self.dev, dtype=dt)  # noqa: E731
        rows = PX.KVRows(t(starts, torch.int64), t(lengths, torch.int32), t(kv_lens, torch.int32),
                         t(self.pages, torch.int32), int(lengths.max(initial=0)), int(kv_lens.max(initial=0)))
        return rows, int((lengths + gap).sum()), starts


def tree_seen(rng, n, shape):
    """[n, n] truth values of what the n nodes of a tree see of it."""
    seen = np.zeros((n, n), bool)
    for i in range(n):
        if shape == "chain":
            parent = i - 1
        elif shape == "star":
            parent = -1
        elif shape == "threads":
            parent = i - 1 if i % max(1, n // 3) else -1
        else:
            parent = int(rng.integers(-1, i)) if i else -1
        if parent >= 0:
            seen[i] = seen[parent]
        seen[i, i] = True
    if shape == "random":
        seen = rng.random((n, n)) < 0.3
    if shape == "empty":
        seen[:] = rng.random((n, n)) < 0.2
        seen[:: 2] = False
    return seen


def words(seen, n_words=None):
    rows, n = seen.shape
    n_words = -(-n // 64) if n_words is None else n_words
    bits = np.zeros((rows, n_words * 64), np.uint8)
    bits[:, :n] = seen
    return np.packbits(bits, axis=1, bitorder="little").view(np.uint64)
