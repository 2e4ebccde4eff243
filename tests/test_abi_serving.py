"""Refusals of the tables', the rotation's and the 4-bit cache's entry points that need no GPU (the fake pointers are
never dereferenced), and the oracle against other ways to the same values."""
import ctypes

import numpy as np
import pytest

from oracle import serving_oracle as S
from paper_2608_24658_amd import parason as P

FAKE = 0x100000


def pool(**kw):
    return P.KvPoolArgs(**dict(dict(free_pages=FAKE, free_count=FAKE, capacity=100), **kw))


def table(**kw):
    return P.KvTableArgs(**dict(dict(n_rows=4, kv_lens=FAKE, pages=FAKE, pages_stride=8, max_pages=8, page_size=16), **kw))


def step(**kw):
    return P.KvStepArgs(**dict(dict(lengths=FAKE, starts=FAKE, row_status=FAKE, positions=FAKE, slots=FAKE, rows=FAKE), **kw))


def tables_workspace(n=4):
    b = ctypes.c_size_t()
    assert P.lib().parason_kv_tables_workspace_size(n, ctypes.byref(b)) == P.OK
    return b.value


BAD_TABLES = [
    (dict(table=dict(n_rows=-1)), P.ERR_SIZE), (dict(table=dict(n_rows=(1 << 24) + 1)), P.ERR_SIZE), (dict(table=dict(max_pages=-1)), P.ERR_SIZE),
    (dict(table=dict(page_size=0)), P.ERR_SIZE), (dict(table=dict(pages_stride=7)), P.ERR_SIZE), (dict(table=dict(pages_stride=-8)), P.ERR_SIZE),
    (dict(table=dict(pages_stride=1 << 60)), P.ERR_SIZE), (dict(pool=dict(capacity=-1)), P.ERR_SIZE), (dict(pool=dict(capacity=1 << 31)), P.ERR_SIZE),
    (dict(pool=dict(free_pages=None)), P.ERR_NULL), (dict(pool=dict(free_count=None)), P.ERR_NULL), (dict(table=dict(kv_lens=None)), P.ERR_NULL),
    (dict(table=dict(pages=None)), P.ERR_NULL), (dict(pool=dict(free_pages=FAKE + 2)), P.ERR_ALIGN), (dict(pool=dict(free_count=FAKE + 1)), P.ERR_ALIGN),
    (dict(table=dict(kv_lens=FAKE + 2)), P.ERR_ALIGN), (dict(table=dict(pages=FAKE + 2)), P.ERR_ALIGN),
]


def test_tables_reject_bad_arguments():
    L, ws = P.lib(), tables_workspace()
    extend = lambda pool_=None, table_=None, lengths=FAKE, n=40, out=None, w=FAKE, b=ws: L.parason_kv_extend(  # noqa: E731
        pool_ or pool(), table_ or table(), lengths, n, out or step(), w, b, None)
    shrink = lambda pool_=None, table_=None, lengths=FAKE, status=FAKE, w=FAKE, b=ws: L.parason_kv_shrink(  # noqa: E731
        pool_ or pool(), table_ or table(), lengths, status, w, b, None)
    for f in (extend, shrink):
        for kw, rc in BAD_TABLES:
            assert f(pool(**kw.get("pool", {})), table(**kw.get("table", {}))) == rc, kw
        assert f(lengths=None) == P.ERR_NULL
        assert f(lengths=FAKE + 2) == P.ERR_ALIGN
        assert f(w=None) == P.ERR_NULL
        assert f(w=FAKE + 16) == P.ERR_ALIGN
        assert f(b=ws - 1) == P.ERR_WORKSPACE
    assert L.parason_kv_extend(None, table(), FAKE, 4, step(), FAKE, ws, None) == P.ERR_NULL
    assert L.parason_kv_extend(pool(), None, FAKE, 4, step(), FAKE, ws, None) == P.ERR_NULL
    assert L.parason_kv_extend(pool(), table(), FAKE, 4, None, FAKE, ws, None) == P.ERR_NULL
    assert L.parason_kv_shrink(None, table(), FAKE, None, FAKE, ws, None) == P.ERR_NULL
    assert L.parason_kv_shrink(pool(), None, FAKE, None, FAKE, ws, None) == P.ERR_NULL
    assert extend(n=-1) == P.ERR_SIZE and extend(n=1 << 31) == P.ERR_SIZE
    for kw, rc in ((dict(lengths=None), P.ERR_NULL), (dict(starts=None), P.ERR_NULL), (dict(lengths=FAKE + 2), P.ERR_ALIGN),
                   (dict(starts=FAKE + 4), P.ERR_ALIGN), (dict(row_status=FAKE + 2), P.ERR_ALIGN), (dict(positions=FAKE + 2), P.ERR_ALIGN),
                   (dict(slots=FAKE + 4), P.ERR_ALIGN), (dict(rows=FAKE + 1), P.ERR_ALIGN)):
        assert extend(out=step(**kw)) == rc, kw
    assert shrink(status=FAKE + 2) == P.ERR_ALIGN
    # nothing to do
    none = table(n_rows=0, kv_lens=None, pages=None)
    assert extend(table_=none, lengths=None, n=0, b=tables_workspace(0)) == P.OK
    assert shrink(table_=none, lengths=None) == P.OK
    b = ctypes.c_size_t()
    for n in (-1, (1 << 24) + 1):
        assert L.parason_kv_tables_workspace_size(n, ctypes.byref(b)) == P.ERR_SIZE
    assert L.parason_kv_tables_workspace_size(4, None) == P.ERR_NULL
    assert tables_workspace(1 << 24) < 200 << 20


def rotate(**kw):
    return P.RotateArgs(**dict(dict(n_tokens=10, n_q_heads=8, n_k_heads=2, head_dim=64, n_turned=64, dtype=P.DTYPE_BF16, flags=0, eps=1e-6,
                                    positions=FAKE, freqs=FAKE, q_weight=FAKE, k_weight=FAKE), **kw))


def heads(**kw):
    return P.HeadsArgs(**dict(dict(q=FAKE, k=FAKE, q_stride_token=640, q_stride_head=64, k_stride_token=640, k_stride_head=64), **kw))


def test_rotation_rejects_bad_arguments():
    L = P.lib()
    b = ctypes.c_size_t()
    assert L.parason_qk_norm_rotate_workspace_size(rotate(), ctypes.byref(b)) == P.OK
    ws = b.value
    forward = lambda r=None, x=None, y=None: L.parason_qk_norm_rotate(r or rotate(), x or heads(), y or heads(), None)  # noqa: E731
    back = lambda r=None, x=None, g=None, y=None, qw=FAKE, kw=FAKE, w=FAKE, n=ws: L.parason_qk_norm_rotate_grad(  # noqa: E731
        r or rotate(), x or heads(), g or heads(), y or heads(), qw, kw, w, n, None)
    for f in (forward, back):
        for kw, rc in [
            (dict(n_tokens=-1), P.ERR_SIZE), (dict(n_tokens=1 << 31), P.ERR_SIZE), (dict(n_q_heads=-1), P.ERR_SIZE),
            (dict(n_k_heads=P.KV_MAX_HEADS + 1), P.ERR_SIZE), (dict(head_dim=0), P.ERR_SIZE), (dict(head_dim=24), P.ERR_SIZE),
            (dict(head_dim=272), P.ERR_SIZE), (dict(n_turned=80), P.ERR_SIZE), (dict(n_turned=8), P.ERR_SIZE), (dict(n_turned=-16), P.ERR_SIZE),
            (dict(dtype=P.DTYPE_FP8), P.ERR_PARAM), (dict(flags=2), P.ERR_PARAM), (dict(eps=0.0), P.ERR_PARAM), (dict(eps=-1.0), P.ERR_PARAM),
            (dict(eps=float("nan")), P.ERR_PARAM), (dict(eps=float("inf")), P.ERR_PARAM), (dict(positions=None), P.ERR_NULL),
            (dict(freqs=None), P.ERR_NULL), (dict(positions=FAKE + 2), P.ERR_ALIGN), (dict(freqs=FAKE + 4), P.ERR_ALIGN),
            (dict(q_weight=FAKE + 1), P.ERR_ALIGN), (dict(dtype=P.DTYPE_F32, k_weight=FAKE + 2), P.ERR_ALIGN),
        ]:
            assert f(rotate(**kw)) == rc, kw
        for kw, rc in [
            (dict(q=None), P.ERR_NULL), (dict(k=None), P.ERR_NULL), (dict(q=FAKE + 1), P.ERR_ALIGN), (dict(k=FAKE + 1), P.ERR_ALIGN),
            (dict(q_stride_token=1 << 60), P.ERR_SIZE), (dict(k_stride_token=-(1 << 60)), P.ERR_SIZE), (dict(q_stride_head=1 << 60), P.ERR_SIZE),
            (dict(k_stride_head=1 << 60), P.ERR_SIZE),
        ]:
            assert f(x=heads(**kw)) == rc, kw
            assert f(y=heads(**kw)) == rc, kw
    assert back(g=heads(q=None)) == P.ERR_NULL
    assert back(qw=FAKE + 2) == P.ERR_ALIGN and back(kw=FAKE + 2) == P.ERR_ALIGN
    assert back(w=None) == P.ERR_NULL and back(w=FAKE + 8) == P.ERR_ALIGN and back(n=ws - 1) == P.ERR_WORKSPACE
    assert L.parason_qk_norm_rotate(None, heads(), heads(), None) == P.ERR_NULL
    assert L.parason_qk_norm_rotate(rotate(), None, heads(), None) == P.ERR_NULL
    assert L.parason_qk_norm_rotate(rotate(), heads(), None, None) == P.ERR_NULL
    assert L.parason_qk_norm_rotate_grad(rotate(), heads(), None, heads(), None, None, FAKE, ws, None) == P.ERR_NULL
    assert L.parason_qk_norm_rotate_workspace_size(rotate(), None) == P.ERR_NULL
    assert L.parason_qk_norm_rotate_workspace_size(rotate(head_dim=17), ctypes.byref(b)) == P.ERR_SIZE
    # nothing to do
    assert forward(rotate(n_tokens=0, positions=None), heads(q=None, k=None), heads(q=None, k=None)) == P.OK
    assert forward(rotate(n_q_heads=0, n_k_heads=0)) == P.OK


def cache(**kw):
    a = dict(k=FAKE, v=FAKE, k_scale=FAKE + 1, v_scale=FAKE + 3, n_pages=10, stride_page=16 * 8 * 128, stride_slot=128, stride_head=16 * 128,
             scale_stride_page=16 * 8 * 4, scale_stride_slot=4, scale_stride_head=64, page_size=16, n_heads=8, head_dim=128, dtype=P.DTYPE_FP4)
    a.update(kw)
    return P.KvCacheArgs(**a)


def rows(**kw):
    a = dict(n_rows=4, n_tokens=40, starts=FAKE, lengths=FAKE, kv_lens=FAKE, pages=FAKE, pages_stride=8, max_pages=8, max_length=10,
             max_kv_len=100)
    a.update(kw)
    return P.KvRowsArgs(**a)


def test_4_bit_caches_reject_bad_arguments():
    L = P.lib()
    b = ctypes.c_size_t()
    calls = [lambda c: L.parason_kv_write(c, rows(), FAKE, FAKE, P.DTYPE_BF16, 1024, 128, None, None),
             lambda c: L.parason_kv_read(c, rows(), FAKE, FAKE, P.DTYPE_BF16, 1024, 128, None, None),
             lambda c: L.parason_tree_attention_workspace_size(c, rows(), 32, ctypes.byref(b))]
    for f in calls:
        for kw, rc in [
            (dict(head_dim=16), P.ERR_SIZE), (dict(head_dim=48), P.ERR_SIZE), (dict(head_dim=288), P.ERR_SIZE), (dict(k_scale=None), P.ERR_NULL),
            (dict(v_scale=None), P.ERR_NULL), (dict(k=FAKE + 8), P.ERR_ALIGN), (dict(stride_slot=144), P.ERR_ALIGN), (dict(stride_head=16), P.ERR_ALIGN),
            (dict(stride_page=16), P.ERR_ALIGN), (dict(scale_stride_page=1 << 60), P.ERR_SIZE),
        ]:
            assert f(cache(**kw)) == rc, kw
    assert calls[2](cache()) == P.OK
    # the scales are bytes: any address and strides do; the arrays' own checks come behind them
    assert L.parason_kv_write(cache(), rows(), None, FAKE, P.DTYPE_F32, 1024, 128, None, None) == P.ERR_NULL
    assert L.parason_kv_write(cache(), rows(), FAKE, FAKE, P.DTYPE_FP4, 1024, 128, None, None) == P.ERR_PARAM


def test_binding_refuses_other_tensors():
    torch = pytest.importorskip("torch")
    c = P.kv_alloc(4, 16, 2, 64, torch.float4_e2m1fn_x2, "cpu")
    assert c.k.shape == (4, 16, 2, 32) and c.k_scale.shape == (4, 16, 2, 2) and c.k.stride(3) == 1
    with pytest.raises(ValueError):
        P.kv_alloc(4, 16, 2, 80, torch.float4_e2m1fn_x2, "cpu")
    i32 = lambda *s: torch.zeros(s, dtype=torch.int32)  # noqa: E731
    r = P.KVRows(torch.zeros(1, dtype=torch.int64), i32(1), i32(1), i32(1, 2), 1, 1)
    x, at, f = torch.zeros(1, 2, 64), i32(1), torch.zeros(32, dtype=torch.float64)
    free = P.kv_pool(4, "cpu")
    assert free.free.tolist() == [3, 2, 1, 0] and free.count.tolist() == [4]
    for call in (lambda: P.kv_write(x, x, c, r), lambda: P.kv_read(c, r, 1, torch.float32), lambda: P.tree_attention(x.bfloat16(), c, r),
                 lambda: P.kv_extend(free, i32(1), i32(1), i32(1, 2), 16, 1), lambda: P.kv_shrink(free, i32(1), i32(1), i32(1, 2), 16),
                 lambda: P.qk_norm_rotate(x, x, at, f), lambda: P.qk_norm_rotate_grad(x, x, x, x, at, f)):
        with pytest.raises(TypeError):
            call()


def _gpu_visible():
    try:
        import torch

        return torch.cuda.device_count() > 0
    except Exception:
        return False


@pytest.mark.skipif(_gpu_visible(), reason="with a GPU these calls would pass the device check and launch")
def test_calls_check_the_device_first():
    L, ws = P.lib(), tables_workspace()
    assert L.parason_kv_extend(pool(), table(), FAKE, 40, step(), FAKE, ws, None) == P.ERR_DEVICE
    assert L.parason_kv_extend(pool(), table(n_rows=0), None, 40, step(), FAKE, ws, None) == P.ERR_DEVICE
    assert L.parason_kv_shrink(pool(), table(), FAKE, None, FAKE, ws, None) == P.ERR_DEVICE
    assert L.parason_qk_norm_rotate(rotate(), heads(), heads(), None) == P.ERR_DEVICE
    assert L.parason_qk_norm_rotate_grad(rotate(), heads(), heads(), heads(), None, None, FAKE, 1 << 30, None) == P.ERR_DEVICE
    assert L.parason_kv_write(cache(), rows(), FAKE, FAKE, P.DTYPE_BF16, 1024, 128, None, None) == P.ERR_DEVICE


# ---- the oracle ------------------------------------------------------------------------------------------------------


def test_oracle_4_bit_values():
    """Every value of the grid is its own code, midpoints go to even codes, and the scale is the least that leaves the
    largest value at most 7 times it."""
    x = np.zeros((16, 32), np.float32)
    x[:, 0] = np.concatenate([S.GRID4, -S.GRID4])
    x[:, 1] = 6.0  # the scale is 1
    codes, s = S.quantise4(x)
    assert np.all(s == 127) and codes[:, 0].tolist() == list(range(16))
    mid = np.zeros((7, 32), np.float32)
    mid[:, 0], mid[:, 1] = (S.GRID4[1:] + S.GRID4[:-1]) / 2, 6.0
    assert S.quantise4(mid)[0][:, 0].tolist() == [0, 2, 2, 4, 4, 6, 6]
    for top, byte, code in ((7.0, 127, 7), (np.nextafter(np.float32(7), np.float32(8)), 128, 6), (3.5, 126, 7), (1e-38, 7, 0), (0.0, 7, 0),
                            (3.4e38, 252, 7), (-1e30, 0, 0)):
        y = np.zeros(32, np.float32)
        y[5] = top
        c, b = S.quantise4(y)
        if byte:
            assert b[0] == byte and c[5] == code, top
        v = S.values4(c, b)
        assert abs(v[5] - top) <= abs(top) / 7 + 2.0 ** -121 or top == np.float32(3.4e38)
    for bad in (np.nan, np.inf):
        y = np.ones((1, 64), np.float32)
        y[0, 40] = bad
        c, b = S.quantise4(y)
        assert b.tolist() == [[125, 255]] and np.isnan(S.values4(c, b)[0, 32:]).all() and np.all(S.values4(c, b)[0, :32] == 1)
    codes = np.random.default_rng(0).integers(0, 16, (3, 64)).astype(np.uint8)
    assert np.array_equal(S.unpack4(S.pack4(codes)), codes)


def test_oracle_tables():
    """A shrink to the lengths before undoes an extend; pages never have two owners."""
    rng = np.random.default_rng(3)
    page, n, per = 4, 9, 6
    kv = rng.integers(0, 9, n).astype(np.int32)
    order = rng.permutation(60).astype(np.int32)
    pages, at = np.full((n, per), -1, np.int32), 0
    for i in range(n):
        k = -(-int(kv[i]) // page)
        pages[i, :k] = order[at: at + k]
        at += k
    free = np.full(60, -1, np.int32)
    free[: 60 - at] = order[at:]
    count = 60 - at
    before = kv.copy(), pages.copy(), free.copy(), count
    lengths = rng.integers(0, 12, n).astype(np.int32)
    count, out = S.extend(free, count, kv, pages, lengths, page, int(lengths.sum()) + 2)
    held = pages[pages >= 0].tolist() + free[:count].tolist()
    assert sorted(held) == list(range(60)) and np.array_equal(out["lengths"], lengths) and out["rows"][-1] == -1
    good = out["rows"] >= 0
    assert np.array_equal(out["slots"][good], pages[out["rows"][good], out["positions"][good] // page] * page + out["positions"][good] % page)
    status = np.zeros(n, np.uint32)
    count = S.shrink(free, count, kv, pages, before[0], page, status)
    assert np.array_equal(kv, before[0]) and np.array_equal(pages, before[1]) and np.array_equal(free, before[2]) and count == before[3]
    assert not status.any()


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("dim,turned", [(16, 16), (48, 32), (32, 0)])
def test_oracle_gradients_against_differences(dim, turned, interleaved):
    """The formula's gradients against central differences of the formula: its third derivative over its first is at most
    some hundreds here (r changes by x / (dim mean x^2)), so steps of 1e-5 leave 1e-7."""
    rng = np.random.default_rng(dim + turned)
    x, dy, w = rng.standard_normal((3, 2, dim)), rng.standard_normal((3, 2, dim)), rng.standard_normal(dim)
    at, freqs = np.array([0, -1, 70000]), 1.0 / 10 ** (4 * np.arange(turned // 2) / max(1, turned // 2))
    f = lambda x, w: (S.rotate(x, w, at, freqs, 1e-6, interleaved)[0] * dy).sum()  # noqa: E731
    dx, dw, _, _ = S.rotate_grad(x, dy, w, at, freqs, 1e-6, interleaved)
    assert np.all(dx[1] == 0)
    for i in np.ndindex(x.shape):
        e = np.zeros(x.shape)
        e[i] = 1e-5
        assert abs((f(x + e, w) - f(x - e, w)) / 2e-5 - dx[i]) < 1e-7 * max(1, np.abs(dy).max() * dim)
    for d in range(dim):
        e = np.zeros(dim)
        e[d] = 1e-5
        assert abs((f(x, w + e) - f(x, w - e)) / 2e-5 - dw[d]) < 1e-7 * dim


def test_oracle_rotation_against_complex_numbers():
    rng = np.random.default_rng(0)
    x, at, freqs = rng.standard_normal((5, 3, 32)), np.array([0, 1, 17, 100003, 7]), rng.random(8)
    y, _ = S.rotate(x, None, at, freqs, 1e-30, True)
    n = x / np.sqrt((x ** 2).mean(-1, keepdims=True))
    z = (n[..., 0:16:2] + 1j * n[..., 1:16:2]) * np.exp(1j * at[:, None, None] * freqs)
    assert np.allclose(y[..., 0:16:2], z.real) and np.allclose(y[..., 1:16:2], z.imag) and np.allclose(y[..., 16:], n[..., 16:])
    y, _ = S.rotate(x, None, at, freqs, 1e-30, False)
    z = (n[..., :8] + 1j * n[..., 8:16]) * np.exp(1j * at[:, None, None] * freqs)
    assert np.allclose(y[..., :8], z.real) and np.allclose(y[..., 8:16], z.imag)
