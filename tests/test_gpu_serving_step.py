"""The serving operators together, as a step uses them: room for the new tokens, their keys and queries normed and turned
by the positions that the tables give, the keys into a 4-bit cache, and the attention over it; eagerly, on another stream,
in a graph that is replayed step after step, and with tokens that belong to nobody."""
import numpy as np
import pytest

from gpu_util import log
from oracle import decoding_oracle as D
from oracle import serving_oracle as S
from paper_2608_24658_amd import parason as PX

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

HEADS, GROUP, DIM, PAGE, MAX_PAGES = 2, 4, 64, 8, 40


@pytest.fixture(scope="module")
def dev():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    return torch.device("cuda:0")


class Engine:
    """A cache, its pool and the rows' tables; the oracle keeps every row's keys and values as the cache holds them."""

    def __init__(self, dev, rows, n_pages, dtype=torch.float4_e2m1fn_x2, page=PAGE):
        self.dev, self.rows, self.page = dev, rows, page
        self.cache = PX.kv_alloc(n_pages, page, HEADS, DIM, dtype, dev)
        self.pool = PX.kv_pool(n_pages, dev)
        self.kv_lens = torch.zeros(rows, dtype=torch.int32, device=dev)
        self.pages = torch.full((rows, MAX_PAGES), -1, dtype=torch.int32, device=dev)
        self.freqs = 1.0 / 1e4 ** (torch.arange(DIM // 2, dtype=torch.float64, device=dev) / (DIM // 2))
        gen = torch.Generator(device=dev).manual_seed(5)
        self.w = (1 + 0.3 * torch.randn(2, DIM, generator=gen, device=dev)).bfloat16()

    def step(self, qkv, lengths, max_length, max_kv_len):
        """One step of packed projections [tokens, heads, dim] for rows with `lengths` new tokens."""
        q_heads = HEADS * GROUP
        q, k, v = qkv[:, :q_heads], qkv[:, q_heads: q_heads + HEADS], qkv[:, q_heads + HEADS:]
        at = PX.kv_extend(self.pool, lengths, self.kv_lens, self.pages, self.page, qkv.shape[0])
        PX.qk_norm_rotate(q, k, at["positions"], self.freqs, *self.w, out=(q, k))
        rows = PX.KVRows(at["starts"], at["lengths"], self.kv_lens, self.pages, max_length, max_kv_len)
        PX.kv_write(k, v, self.cache, rows)
        return PX.tree_attention(q, self.cache, rows), at


def expect(q, k, held, n):
    """Bounds of one row's results from what its cache holds: (out, tolerance)."""
    kk, vv = held
    return D.attention(q, kk, vv, D.visible(kk.shape[0], n), DIM ** -0.5, 7, 7)[0::2]


@pytest.mark.parametrize("graph", [False, True])
def test_steps(dev, graph):
    """A prompt for each row, then single tokens, with rows that wait and tokens to spare.  After each step every row's
    attention is checked against the oracle over the keys that the oracle rotates and quantises itself; a key that lies on
    the border of two codes may take either (float32 against 64 bits), so the oracle goes on with the cache's own codes
    where they are one step apart, which few may be."""
    log("case serving steps, graph %s" % graph)
    rng = np.random.default_rng(0)
    rows, spare = 5, 3
    E = Engine(dev, rows, 60)
    held = [[np.zeros((0, HEADS, DIM)), np.zeros((0, HEADS, DIM))] for _ in range(rows)]
    g = static = None
    for n_step in range(6):
        lengths = rng.integers(1, 40, rows) if n_step == 0 else (rng.random(rows) < 0.8).astype(np.int64)
        total = int(lengths.sum()) + spare if n_step == 0 else rows + spare
        x = torch.randn(total, HEADS * (GROUP + 2), DIM, device=dev).bfloat16()
        given = x.clone()
        d_len = torch.as_tensor(lengths).to(device=dev, dtype=torch.int32)
        if n_step == 0 or not graph:
            out, at = E.step(x, d_len, 40, 200)
        else:
            if g is None:
                static = dict(x=x.clone(), lengths=d_len.clone())
                g = torch.cuda.CUDAGraph()
                torch.cuda.synchronize()
                with torch.cuda.graph(g):
                    static["out"], static["at"] = E.step(static["x"], static["lengths"], 1, 200)
            static["x"].copy_(x)
            static["lengths"].copy_(d_len)
            g.replay()
            torch.cuda.synchronize()
            out, at, x = static["out"], static["at"], static["x"]
        assert at["status"].tolist() == [0] * rows and at["lengths"].tolist() == lengths.tolist()
        positions = at["positions"].cpu().numpy()
        freqs = E.freqs.cpu().numpy()
        host = given.double().cpu().numpy()
        q_heads = HEADS * GROUP
        want = [S.rotate(host[:, a:b], E.w[i].double().cpu().numpy(), positions, freqs, 1e-6, False)
                for i, (a, b) in enumerate(((0, q_heads), (q_heads, q_heads + HEADS)))]
        for i, (a, b) in enumerate(((0, q_heads), (q_heads, q_heads + HEADS))):
            y = x[:, a:b].double().cpu().numpy()
            assert np.all(np.abs(y - want[i][0]) <= want[i][1] + (np.abs(want[i][0]) + want[i][1]) * 2.0 ** -8 + 2.0 ** -134)
        qh, kh = x[:, :q_heads].double().cpu().numpy(), x[:, q_heads: q_heads + HEADS].float().cpu().numpy()
        vh = given[:, q_heads + HEADS:].float().cpu().numpy()
        got = out.double().cpu().numpy()
        start = 0
        for i, n in enumerate(lengths):
            new = slice(start, start + n)
            start += n
            for w, src in enumerate((kh, vh)):
                if n:
                    codes = S.quantise4(src[new])
                    held[i][w] = np.concatenate([held[i][w], S.values4(*codes).astype(np.float64)])
            assert positions[new].tolist() == list(range(held[i][0].shape[0] - n, held[i][0].shape[0]))
            if n:
                o, tol = expect(qh[new], None, held[i], int(n))
                assert np.all(np.abs(got[new] - o) <= tol), (n_step, i)
        assert np.all(positions[start:] == -1) and (x[start:, : q_heads + HEADS] == 0).all()
    # what is left is whole: no page has two owners, and all come back
    owned = E.pages[E.pages >= 0].tolist() + E.pool.free[: int(E.pool.count)].tolist()
    assert sorted(owned) == list(range(60))
    PX.kv_shrink(E.pool, torch.zeros_like(E.kv_lens), E.kv_lens, E.pages, PAGE)
    assert int(E.pool.count) == 60 and (E.pages == -1).all() and (E.kv_lens == 0).all()


def test_refused_drafts(dev):
    """Draft tokens are written, most are refused and taken back, and what follows is as if they had never been."""
    log("case refused drafts")
    results = []
    for draft in (False, True):
        E = Engine(dev, 3, 40, torch.bfloat16)
        gen = torch.Generator(device=dev).manual_seed(1)
        i32 = lambda *a: torch.tensor(a, dtype=torch.int32, device=dev)  # noqa: E731
        make = lambda n: torch.randn(n, HEADS * (GROUP + 2), DIM, generator=gen, device=dev).bfloat16()  # noqa: E731
        first, drafts, last = make(60), make(36), make(3)
        E.step(first, i32(30, 7, 23), 30, 200)
        if draft:
            before = E.kv_lens.clone(), E.pages.clone(), E.pool.free.clone(), E.pool.count.clone()
            E.step(drafts, i32(20, 9, 7), 20, 200)
            PX.kv_shrink(E.pool, before[0], E.kv_lens, E.pages, PAGE)
            for a, b in zip(before, (E.kv_lens, E.pages, E.pool.free, E.pool.count)):
                assert torch.equal(a, b)
        results.append(E.step(last, i32(1, 1, 1), 1, 200)[0])
    assert torch.equal(*results)


def test_rows_that_get_no_pages(dev):
    """A pool that runs dry: the rows that are not served write nothing, see nothing, and the others are whole."""
    log("case dry pool")
    E = Engine(dev, 4, 5)
    x = torch.randn(60, HEADS * (GROUP + 2), DIM, device=dev).bfloat16()
    lengths = torch.tensor([20, 8, 20, 12], dtype=torch.int32, device=dev)
    y = x.clone()
    out, at = E.step(y, lengths, 20, 200)
    assert at["status"].tolist() == [0, 0, PX.KV_NO_PAGES, PX.KV_NO_PAGES] and at["lengths"].tolist() == [20, 8, 0, 0]
    assert E.kv_lens.tolist() == [20, 8, 0, 0] and int(E.pool.count) == 1 and (at["slots"][28:] == -1).all()
    alone = Engine(dev, 2, 5)
    z = x[:28].clone()
    want, _ = alone.step(z, lengths[:2].contiguous(), 20, 200)
    assert torch.equal(out[:28], want)
