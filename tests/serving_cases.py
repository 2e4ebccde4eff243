"""Caches in 4 bits and rows' tables for the tests of the serving operators."""
import numpy as np

import decoding_cases as C
from oracle import serving_oracle as S
from paper_2608_24658_amd import parason as PX


class Paged4(C.Paged):
    """decoding_cases.Paged with a 4-bit cache (kind "fp4")."""

    def __init__(self, dev, kv_lens, page, heads, dim, kind, seed, layout="heads", spare=3, pad=0, extra_slots=0):
        import torch

        assert kind == "fp4"
        super().__init__("cpu", kv_lens, page, heads, dim, "bf16", seed, layout, spare, pad, extra_slots)
        self.dev, self.kind = dev, kind
        lead = dict(heads=(self.n_pages, heads, page), slots=(self.n_pages, page, heads))[layout]
        swap = (0, 2, 1, 3) if layout == "heads" else (0, 1, 2, 3)
        # what no one has written: scales that make everything NaN (`pad`: values between a head and the next)
        made = [torch.full(lead + ((dim + 2 * pad) // n,), 255, dtype=torch.uint8).to(dev) for n in (2, 2, 32, 32)]
        types = [torch.float4_e2m1fn_x2] * 2 + [torch.float8_e8m0fnu] * 2
        made = [x.view(t).permute(swap)[..., : dim // n] for x, t, n in zip(made, types, (2, 2, 32, 32))]
        self.kv, self.scales = made[:2], made[2:]
        self.cache = PX.KVCache(*made)

    def fill(self, values_of):
        import torch

        host = [t.view(torch.uint8).cpu().clone() for t in self.kv + self.scales]
        self.held = []
        for i, n in enumerate(self.kv_lens):
            x = np.asarray(values_of(i, int(n)), np.float32)
            pg, slot = self.place(i, np.arange(int(n)))
            held = []
            for w in range(2):
                codes, s = S.quantise4(x[w])
                host[w][pg, slot] = torch.from_numpy(S.pack4(codes))
                host[2 + w][pg, slot] = torch.from_numpy(s)
                held.append(S.values4(codes, s).astype(np.float64))
            self.held.append(held)
        for t, h in zip(self.kv + self.scales, host):
            t.view(torch.uint8).copy_(h)
        return self


class Tables:
    """Rows on random pages of a pool, on the host and on the device."""

    def __init__(self, dev, kv_lens, page, max_pages, seed=0, spare=5, pad=0):
        import torch

        rng = np.random.default_rng(seed)
        self.page, self.kv_lens = page, np.asarray(kv_lens, np.int32)
        need = np.maximum(-(-self.kv_lens // page), 0)
        total = int(need.sum()) + spare
        order = rng.permutation(total).astype(np.int32)
        self.pages = np.full((len(kv_lens), max_pages), -1, np.int32)
        at = 0
        for i, k in enumerate(need):
            self.pages[i, :k] = order[at: at + k]
            at += int(k)
        self.free = np.full(total, -9, np.int32)
        self.free[: total - at] = order[at:]
        self.count = total - at
        t = lambda a: torch.as_tensor(np.array(a)).to(device=dev, dtype=torch.int32)  # noqa: E731
        self.d_lens, self.d_free, self.d_count = t(self.kv_lens), t(self.free), t([self.count])
        wide = torch.full((len(kv_lens), max_pages + pad), -77, dtype=torch.int32, device=dev)
        self.d_wide, self.d_pages = wide, wide[:, :max_pages]
        self.d_pages.copy_(t(self.pages))
        self.pool = PX.KVPool(self.d_free, self.d_count)

    def check(self):
        got = [t.cpu().numpy() for t in (self.d_lens, self.d_pages, self.d_free, self.d_count)]
        for name, g, w in zip(("kv_lens", "pages", "free", "count"), got, (self.kv_lens, self.pages, self.free, [self.count])):
            assert np.array_equal(g, w), (name, np.nonzero(g != w))
        assert (self.d_wide[:, self.pages.shape[1]:] == -77).all()

    def extend(self, lengths, n_tokens=None):
        import torch

        lengths = np.asarray(lengths, np.int32)
        n_tokens = int(np.maximum(lengths, 0).sum()) if n_tokens is None else n_tokens
        d = torch.as_tensor(lengths).to(self.d_lens.device)
        got = PX.kv_extend(self.pool, d, self.d_lens, self.d_pages, self.page, n_tokens)
        self.count, want = S.extend(self.free, self.count, self.kv_lens, self.pages, lengths, self.page, n_tokens)
        for k, w in want.items():
            g = got[k].cpu().numpy()
            assert np.array_equal(g, w.view(g.dtype)), (k, np.nonzero(g != w.view(g.dtype)), g[:20], w[:20])
        self.check()
        return got, want

    def shrink(self, new_lens):
        import torch

        new_lens = np.asarray(new_lens, np.int32)
        status, want = torch.zeros(len(new_lens), dtype=torch.int32, device=self.d_lens.device), np.zeros(len(new_lens), np.int64)
        PX.kv_shrink(self.pool, torch.as_tensor(new_lens).to(self.d_lens.device), self.d_lens, self.d_pages, self.page, status=status)
        self.count = S.shrink(self.free, self.count, self.kv_lens, self.pages, new_lens, self.page, want)
        assert np.array_equal(status.cpu().numpy(), want)
        self.check()
        return want
