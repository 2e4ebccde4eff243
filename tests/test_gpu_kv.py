"""The paged cache's write and read on the GPU against the oracle: codes, scales and values bit for bit (each is one
correctly rounded float32 operation or copy on both sides), everything that the call does not own untouched."""
import numpy as np
import pytest

from decoding_cases import KINDS, Paged, torch_type
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


def bits(t):
    """A tensor's bytes on the host (NaN compares by pattern)."""
    t = t.detach().cpu().contiguous()
    return t.view(torch.uint8).numpy() if t.element_size() == 1 else t.view({2: torch.int16, 4: torch.int32}[t.element_size()]).numpy()


def given_types(kind):
    return {"bf16": ("bf16", "fp32"), "fp16": ("fp16", "fp32")}.get(kind, ("bf16", "fp16", "fp32"))


SHAPES = [
    # lengths, positions before them, page, heads, dim, layout
    ([1], [0], 16, 1, 128, "heads"),
    ([1, 1, 1, 0, 1], [0, 15, 16, 40, 1000], 16, 8, 128, "heads"),
    ([5, 0, 37, 130], [0, 0, 27, 3], 24, 3, 64, "slots"),
    ([300, 1], [0, 511], 1, 2, 80, "heads"),
    ([33, 64], [100, 1], 128, 5, 16, "slots"),
    ([7, 90], [2, 10], 100, 16, 256, "heads"),
    ([11, 2], [2, 10], 8, 2, 192, "slots"),
]


@pytest.mark.parametrize("kind,given", [(k, g) for k in KINDS for g in given_types(k)])
@pytest.mark.parametrize("shape", range(len(SHAPES)))
def test_write_then_read(dev, shape, kind, given):
    lengths, before, page, heads, dim, layout = SHAPES[shape]
    log("case kv %s given %s shape %d" % (kind, given, shape))
    lengths = np.array(lengths)
    P = Paged(dev, np.array(before) + lengths, page, heads, dim, kind, seed=shape, layout=layout)
    rng = np.random.default_rng(100 + shape)
    rows, total, starts = P.rows(lengths, gap=2)
    x = rng.standard_normal((2, total, heads, dim)).astype(np.float32) * 10.0 ** rng.integers(-6, 6, (2, total, heads, 1))
    x[:, :, 0, :3] = 0.0
    if total > 4:
        x[:, 3] = 0.0  # a head of zeros
        x[0, 2, 0, 5], x[1, 4, heads - 1, 1] = np.inf, np.nan
    x = torch.as_tensor(x.astype(np.float32)).to(torch_type(given))
    # strides other than the tight ones, and arrays that begin in the middle of 16 bytes
    flat = torch.zeros(2, total, heads, dim + 3 * (shape % 2), dtype=x.dtype, device=dev)[..., :dim]
    flat.copy_(x)
    k, v = flat if shape % 3 else (flat[0].clone(), flat[1].clone())
    cache_before = [bits(t).copy() for t in P.kv + P.scales]
    status = torch.zeros(len(lengths), dtype=torch.int32, device=dev)
    PX.kv_write(k, v, P.cache, rows, status=status)
    expect = [c.copy() for c in cache_before]
    for i, n in enumerate(lengths):
        pg, slot = P.place(i, before[i] + np.arange(n))
        for w in range(2):
            part = x[w, starts[i]: starts[i] + n].float()
            if P.scales:
                codes, s = D.quantise(part.numpy(), kind)
                expect[w][pg, slot] = codes.view(np.uint8)
                expect[2 + w][pg, slot] = s.view(np.int32)
            else:
                expect[w][pg, slot] = part.to(torch_type(kind)).view(torch.int16).numpy()
    for name, e, t in zip(("k", "v", "k_scale", "v_scale"), expect, P.kv + P.scales):
        got = bits(t)
        if not P.scales:  # NaN payloads are not specified
            e, got = (torch.from_numpy(a).view(torch_type(kind)).float().numpy() for a in (e, got))
            assert np.array_equal(e, got, equal_nan=True), name
        elif name.endswith("scale"):
            assert np.array_equal(e.view(np.float32), got.view(np.float32), equal_nan=True), name
        else:
            assert np.array_equal(e, got), (name, np.nonzero(e != got))
    # read everything back, into every type
    for to in ("fp32", "bf16", "fp16"):
        all_rows, n, begin = P.rows(P.kv_lens, gap=1)
        out = torch.full((2, n, heads, dim), 77.0, dtype=torch_type(to), device=dev)
        got = PX.kv_read(P.cache, all_rows, n, torch_type(to), out=(out[0], out[1]), status=status)
        for w in range(2):
            want = torch.full((n, heads, dim), 77.0, dtype=torch_type(to))
            for i, m in enumerate(P.kv_lens):
                pg, slot = P.place(i, np.arange(m))
                if P.scales:
                    val = D.values(expect[w][pg, slot], expect[2 + w][pg, slot].view(np.float32), kind)
                    val = torch.from_numpy(val)
                else:
                    val = torch.from_numpy(expect[w][pg, slot]).view(torch_type(kind)).float()
                want[begin[i]: begin[i] + m] = val.to(torch_type(to))
            assert torch.equal(torch.nan_to_num(want.float(), nan=12345.0), torch.nan_to_num(got[w].cpu().float(), nan=12345.0)), (to, w)
    assert status.cpu().tolist() == [0] * len(lengths)


def test_rows_and_pages_that_are_bad(dev):
    """Bad rows and pages are reported, nothing of them is written, and the rows beside them are whole."""
    P = Paged(dev, [20, 20, 20, 20, 20, 20], 8, 2, 64, "fp8", seed=3)
    rows, total, starts = P.rows([4] * 6)
    x = torch.randn(total, 2, 64).to(dev)
    lengths, kv, st = rows.lengths.clone(), rows.kv_lens.clone(), rows.starts.clone()
    lengths[1] = -1
    kv[2] = 3            # fewer than the new tokens
    st[3] = total - 2    # reaches behind the arrays
    kv[4] = 1 << 20      # more than the bound
    pages = rows.pages.clone()
    pages[5, 2] = 10 ** 6  # positions 16 .. 19
    rows = rows._replace(lengths=lengths, kv_lens=kv, starts=st, pages=pages)
    before = [bits(t).copy() for t in P.kv + P.scales]
    status = torch.zeros(6, dtype=torch.int32, device=dev)
    PX.kv_write(x, x, P.cache, rows, status=status)
    assert status.cpu().tolist() == [0, PX.KV_BAD_ROW, PX.KV_BAD_ROW, PX.KV_BAD_ROW, PX.KV_BAD_ROW, PX.KV_BAD_PAGE]
    codes, s = D.quantise(x[starts[0]: starts[0] + 4].cpu().numpy(), "fp8")
    pg, slot = P.place(0, 16 + np.arange(4))
    for w in range(2):
        before[w][pg, slot] = codes
        before[2 + w][pg, slot] = s.view(np.int32)
    for b, t in zip(before, P.kv + P.scales):
        assert np.array_equal(b, bits(t))
    out = torch.full((2, total, 2, 64), 5.0, device=dev)
    PX.kv_read(P.cache, rows, total, torch.float32, out=(out[0], out[1]))
    got = out.cpu()
    assert torch.equal(got[0, :4], torch.from_numpy(D.values(codes, s, "fp8")))
    assert torch.all(got[:, 4:20] == 5.0) and torch.isnan(got[:, 20:24]).all()


def test_offsets_beyond_32_bits(dev):
    """Pages whose elements lie behind 2^32 of the pool's first."""
    n_pages, page, heads, dim = 270_000, 16, 4, 256
    cache = PX.kv_alloc(n_pages, page, heads, dim, torch.float16, dev)
    far = cache.k.numel() > 1 << 32 and cache.k.stride(0) == page * heads * dim
    assert far
    pages = torch.tensor([[n_pages - 1, 0, n_pages - 2]], dtype=torch.int32, device=dev)
    one = lambda v, dt: torch.tensor([v], dtype=dt, device=dev)  # noqa: E731
    rows = PX.KVRows(one(0, torch.int64), one(40, torch.int32), one(40, torch.int32), pages, 40, 40)
    x = torch.randn(2, 40, heads, dim, device=dev, dtype=torch.float16)
    PX.kv_write(x[0], x[1], cache, rows)
    k, v = PX.kv_read(cache, rows, 40, torch.float16)
    same = torch.equal(k, x[0]) and torch.equal(v, x[1])
    assert same
    same = torch.equal(cache.k[n_pages - 1], x[0, :16]) and torch.equal(cache.v[n_pages - 2, :8], x[1, 32:])
    assert same
    same = int((cache.k != 0).sum()) == int((x[0] != 0).sum())
    assert same


def test_empty_calls(dev):
    cache = PX.kv_alloc(2, 4, 2, 32, torch.int8, dev)
    none = lambda dt: torch.empty(0, dtype=dt, device=dev)  # noqa: E731
    rows = PX.KVRows(none(torch.int64), none(torch.int32), none(torch.int32), torch.empty(0, 0, dtype=torch.int32, device=dev), 0, 0)
    PX.kv_write(torch.empty(0, 2, 32, device=dev), torch.empty(0, 2, 32, device=dev), cache, rows)
    k, v = PX.kv_read(cache, rows, 0, torch.float32)
    assert k.shape == (0, 2, 32)
