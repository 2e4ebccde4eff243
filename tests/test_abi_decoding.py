"""Refusals of the cache, tree attention and beam entry points that need no GPU: every call below fails a host check
before the first HIP call (the fake pointers are never dereferenced).  And the oracle's 8-bit codes against torch's."""
import ctypes

import numpy as np
import pytest

from oracle import decoding_oracle as D
from paper_2608_24658_amd import parason as P

FAKE = 0x100000


def cache(**kw):
    a = dict(k=FAKE, v=FAKE, k_scale=FAKE, v_scale=FAKE, n_pages=10, stride_page=16 * 8 * 128, stride_slot=128, stride_head=16 * 128,
             scale_stride_page=128, scale_stride_slot=1, scale_stride_head=16, page_size=16, n_heads=8, head_dim=128, dtype=P.DTYPE_FP8)
    a.update(kw)
    return P.KvCacheArgs(**a)


def rows(**kw):
    a = dict(n_rows=4, n_tokens=40, starts=FAKE, lengths=FAKE, kv_lens=FAKE, pages=FAKE, pages_stride=8, max_pages=8, max_length=10,
             max_kv_len=100)
    a.update(kw)
    return P.KvRowsArgs(**a)


def tree(**kw):
    a = dict(q=FAKE, out=FAKE, lse=FAKE, q_stride_token=4096, q_stride_head=128, out_stride_token=4096, out_stride_head=128, mask=FAKE,
             mask_stride=2, tree_lens=FAKE, mask_words=2, n_q_heads=32, dtype=P.DTYPE_BF16, scale=0.1)
    a.update(kw)
    return P.TreeArgs(**a)


BAD_CACHES = [
    (dict(dtype=P.DTYPE_F32), P.ERR_PARAM), (dict(dtype=9), P.ERR_PARAM), (dict(n_pages=-1), P.ERR_SIZE), (dict(n_pages=1 << 31), P.ERR_SIZE),
    (dict(page_size=0), P.ERR_SIZE), (dict(n_heads=0), P.ERR_SIZE), (dict(n_heads=P.KV_MAX_HEADS + 1), P.ERR_SIZE),
    (dict(head_dim=0), P.ERR_SIZE), (dict(head_dim=24), P.ERR_SIZE), (dict(head_dim=P.KV_MAX_DIM + 16), P.ERR_SIZE),
    (dict(stride_page=1 << 60), P.ERR_SIZE), (dict(scale_stride_slot=-(1 << 60)), P.ERR_SIZE), (dict(k=None), P.ERR_NULL),
    (dict(v=None), P.ERR_NULL), (dict(k_scale=None), P.ERR_NULL), (dict(v_scale=None), P.ERR_NULL), (dict(k=FAKE + 8), P.ERR_ALIGN),
    (dict(v=FAKE + 2), P.ERR_ALIGN), (dict(stride_slot=136), P.ERR_ALIGN), (dict(stride_head=4), P.ERR_ALIGN),
    (dict(dtype=P.DTYPE_BF16, stride_page=12), P.ERR_ALIGN), (dict(v_scale=FAKE + 2), P.ERR_ALIGN),
]
BAD_ROWS = [
    (dict(n_rows=-1), P.ERR_SIZE), (dict(n_tokens=-1), P.ERR_SIZE), (dict(max_pages=-1), P.ERR_SIZE), (dict(max_length=-1), P.ERR_SIZE),
    (dict(max_kv_len=-1), P.ERR_SIZE), (dict(pages_stride=1 << 60), P.ERR_SIZE), (dict(starts=None), P.ERR_NULL),
    (dict(lengths=None), P.ERR_NULL), (dict(kv_lens=None), P.ERR_NULL), (dict(pages=None), P.ERR_NULL), (dict(starts=FAKE + 4), P.ERR_ALIGN),
    (dict(lengths=FAKE + 2), P.ERR_ALIGN), (dict(pages=FAKE + 1), P.ERR_ALIGN),
]


@pytest.mark.parametrize("name", ["parason_kv_write", "parason_kv_read"])
def test_cache_moves_reject_bad_arguments(name):
    fn = getattr(P.lib(), name)
    call = lambda c=None, r=None, k=FAKE, v=FAKE, dt=P.DTYPE_BF16, st=1024, sh=128, status=FAKE: fn(  # noqa: E731
        c or cache(), r or rows(), k, v, dt, st, sh, status, None)
    for kw, rc in BAD_CACHES:
        assert call(c=cache(**kw)) == rc, kw
    for kw, rc in BAD_ROWS:
        assert call(r=rows(**kw)) == rc, kw
    assert fn(None, rows(), FAKE, FAKE, P.DTYPE_BF16, 1024, 128, None, None) == P.ERR_NULL
    assert fn(cache(), None, FAKE, FAKE, P.DTYPE_BF16, 1024, 128, None, None) == P.ERR_NULL
    assert call(dt=P.DTYPE_FP8) == P.ERR_PARAM
    assert call(k=None) == P.ERR_NULL
    assert call(v=FAKE + 1) == P.ERR_ALIGN
    assert call(dt=P.DTYPE_F32, k=FAKE + 2) == P.ERR_ALIGN
    assert call(status=FAKE + 2) == P.ERR_ALIGN
    assert call(st=1 << 60) == P.ERR_SIZE
    assert call(r=rows(max_length=1 << 28)) == P.ERR_SIZE
    # nothing to do
    assert call(r=rows(n_rows=0)) == P.OK
    assert call(r=rows(max_length=0), k=None) == P.OK
    # a 16-bit cache is written from its own type or float32, and read into any
    c = cache(dtype=P.DTYPE_F16, k_scale=None, v_scale=None)
    assert call(c=c, k=None) == (P.ERR_PARAM if name == "parason_kv_write" else P.ERR_NULL)


def test_tree_attention_rejects_bad_arguments():
    size, fn = P.lib().parason_tree_attention_workspace_size, P.lib().parason_tree_attention
    ws = ctypes.c_size_t()
    assert size(cache(), rows(), 32, ctypes.byref(ws)) == P.OK
    assert size(cache(), rows(), 32, None) == P.ERR_NULL
    assert size(cache(), rows(), 30, ctypes.byref(ws)) == P.ERR_SIZE
    assert size(cache(), rows(), 0, ctypes.byref(ws)) == P.ERR_SIZE
    W = 1 << 40
    call = lambda c=None, r=None, t=None, status=FAKE, w=FAKE, n=W: fn(c or cache(), r or rows(), t or tree(), status, w, n, None)  # noqa: E731
    for kw, rc in BAD_CACHES:
        assert call(c=cache(**kw)) == rc, kw
    for kw, rc in BAD_ROWS:
        assert call(r=rows(**kw)) == rc, kw
    for kw, rc in [
        (dict(dtype=P.DTYPE_F32), P.ERR_PARAM), (dict(scale=float("nan")), P.ERR_PARAM), (dict(scale=float("inf")), P.ERR_PARAM),
        (dict(mask=None), P.ERR_PARAM), (dict(n_q_heads=12), P.ERR_SIZE), (dict(n_q_heads=-8), P.ERR_SIZE), (dict(mask_words=-1), P.ERR_SIZE),
        (dict(q_stride_token=1 << 60), P.ERR_SIZE), (dict(out_stride_head=1 << 60), P.ERR_SIZE), (dict(mask_stride=1 << 60), P.ERR_SIZE),
        (dict(q=None), P.ERR_NULL), (dict(out=None), P.ERR_NULL), (dict(q=FAKE + 1), P.ERR_ALIGN), (dict(out=FAKE + 1), P.ERR_ALIGN),
        (dict(lse=FAKE + 2), P.ERR_ALIGN), (dict(mask=FAKE + 4), P.ERR_ALIGN), (dict(tree_lens=FAKE + 2), P.ERR_ALIGN),
    ]:
        assert call(t=tree(**kw)) == rc, kw
    for dt in (P.DTYPE_BF16, P.DTYPE_F16):
        c = cache(dtype=dt, k_scale=None, v_scale=None)
        assert call(c=c, t=tree(dtype=P.DTYPE_BF16 + P.DTYPE_F16 - dt)) == P.ERR_PARAM
    assert fn(cache(), rows(), None, None, FAKE, W, None) == P.ERR_NULL
    assert call(w=None) == P.ERR_NULL
    assert call(w=FAKE + 8) == P.ERR_ALIGN
    assert call(n=0) == P.ERR_WORKSPACE
    assert call(n=ws.value - 1) == P.ERR_WORKSPACE
    assert call(status=FAKE + 1) == P.ERR_ALIGN
    assert call(r=rows(n_rows=0), t=tree(q=None)) == P.OK
    assert call(r=rows(max_length=0), w=None) == P.OK


def test_rows_longer_than_31_bits_can_count():
    """Positions and columns are counted in 32 bits, a tile beyond the last one included."""
    L, ws, over = P.lib(), ctypes.c_size_t(), P.KV_MAX_LEN + 1
    for fn in (L.parason_kv_write, L.parason_kv_read):
        assert fn(cache(), rows(max_kv_len=over), FAKE, FAKE, P.DTYPE_BF16, 1024, 128, None, None) == P.ERR_SIZE
    size = L.parason_tree_attention_workspace_size
    assert size(cache(), rows(max_kv_len=over), 32, ctypes.byref(ws)) == P.ERR_SIZE
    assert size(cache(), rows(max_kv_len=P.KV_MAX_LEN), 32, ctypes.byref(ws)) == P.OK
    assert size(cache(), rows(max_length=P.KV_MAX_LEN // 4), 32, ctypes.byref(ws)) == P.OK
    assert size(cache(), rows(max_length=P.KV_MAX_LEN // 4 + 1), 32, ctypes.byref(ws)) == P.ERR_SIZE
    for n in (1 << 20, (1 << 31) - 1):  # products of sizes that no 64 bits hold among them
        assert size(cache(), rows(n_rows=n, max_length=P.KV_MAX_LEN // 4), 32, ctypes.byref(ws)) == P.ERR_SIZE
    assert L.parason_tree_attention(cache(), rows(max_length=P.KV_MAX_LEN // 4 + 1), tree(), None, FAKE, 1 << 40, None) == P.ERR_SIZE


def test_beam_select_rejects_bad_arguments():
    size, fn = P.lib().parason_beam_workspace_size, P.lib().parason_beam_select
    ws = ctypes.c_size_t()
    assert size(4, 8, 1000, ctypes.byref(ws)) == P.OK and ws.value > 0
    for g, b, v in ((-1, 8, 10), (4, 0, 10), (4, P.BEAM_MAX + 1, 10), (4, 8, 0), (1 << 30, 8, 10), (1, 1, 1 << 31)):
        assert size(g, b, v, ctypes.byref(ws)) == P.ERR_SIZE
    assert size(4, 8, 1000, None) == P.ERR_NULL
    size(4, 8, 1000, ctypes.byref(ws))
    good = dict(logits=FAKE, vocab=1000, stride=1000, dtype=P.DTYPE_BF16, scores=FAKE, states=FAKE, groups=4, beams=8, new=FAKE, parents=FAKE,
                tokens=FAKE, ws=FAKE, n=ws.value, stream=None)
    for kw, rc in [
        (dict(stride=999), P.ERR_SIZE), (dict(stride=1 << 60), P.ERR_SIZE), (dict(dtype=P.DTYPE_FP8), P.ERR_PARAM), (dict(logits=None), P.ERR_NULL),
        (dict(scores=None), P.ERR_NULL), (dict(new=None), P.ERR_NULL), (dict(parents=None), P.ERR_NULL), (dict(tokens=None), P.ERR_NULL),
        (dict(ws=None), P.ERR_NULL), (dict(logits=FAKE + 1), P.ERR_ALIGN), (dict(logits=FAKE + 2, dtype=P.DTYPE_F32), P.ERR_ALIGN),
        (dict(states=FAKE + 8), P.ERR_ALIGN), (dict(scores=FAKE + 2), P.ERR_ALIGN), (dict(ws=FAKE + 16), P.ERR_ALIGN),
        (dict(n=ws.value - 1), P.ERR_WORKSPACE), (dict(groups=0, logits=None), P.OK),
    ]:
        assert fn(*dict(good, **kw).values()) == rc, kw


def test_beam_reorder_rejects_bad_arguments():
    fn = P.lib().parason_beam_reorder
    arr = lambda **kw: (P.BeamArray * 1)(P.BeamArray(**dict(dict(src=FAKE, dst=FAKE + 4096, row_bytes=16, src_stride=16, dst_stride=16), **kw)))  # noqa: E731
    assert fn(FAKE, -1, arr(), 1, None) == P.ERR_SIZE
    assert fn(FAKE, 4, arr(), P.BEAM_ARRAYS + 1, None) == P.ERR_SIZE
    assert fn(FAKE, 4, arr(), -1, None) == P.ERR_SIZE
    assert fn(None, 4, arr(), 1, None) == P.ERR_NULL
    assert fn(FAKE, 4, None, 1, None) == P.ERR_NULL
    assert fn(FAKE + 2, 4, arr(), 1, None) == P.ERR_ALIGN
    assert fn(FAKE, 4, arr(src=None), 1, None) == P.ERR_NULL
    assert fn(FAKE, 4, arr(dst=None), 1, None) == P.ERR_NULL
    assert fn(FAKE, 4, arr(row_bytes=-1), 1, None) == P.ERR_SIZE
    assert fn(FAKE, 4, arr(src_stride=15), 1, None) == P.ERR_SIZE
    assert fn(FAKE, 4, arr(dst_stride=1 << 60), 1, None) == P.ERR_SIZE
    assert fn(None, 0, None, 0, None) == P.OK
    assert fn(FAKE, 4, arr(row_bytes=0, src=None), 1, None) == P.OK


def test_binding_refuses_other_tensors():
    torch = pytest.importorskip("torch")
    c = P.kv_alloc(4, 16, 2, 64, torch.int8, "cpu")
    r = P.KVRows(*(torch.zeros(1, dtype=d) for d in (torch.int64, torch.int32, torch.int32)), torch.zeros(1, 2, dtype=torch.int32), 1, 1)
    x = torch.zeros(1, 2, 64)
    for f in (lambda: P.kv_write(x, x, c, r), lambda: P.kv_read(c, r, 1, torch.float32), lambda: P.tree_attention(x.bfloat16(), c, r),
              lambda: P.beam_select(torch.zeros(4, 9), torch.zeros(4), 2), lambda: P.beam_reorder(torch.zeros(4, dtype=torch.int32), [])):
        with pytest.raises(TypeError):
            f()
    with pytest.raises(TypeError):
        P.kv_alloc(4, 16, 2, 64, torch.float32, "cpu")


def _gpu_visible():
    try:
        import torch

        return torch.cuda.device_count() > 0
    except Exception:
        return False


@pytest.mark.skipif(_gpu_visible(), reason="with a GPU these calls would pass the device check and launch")
def test_calls_check_the_device_first():
    L = P.lib()
    assert L.parason_kv_write(cache(), rows(), FAKE, FAKE, P.DTYPE_BF16, 1024, 128, None, None) == P.ERR_DEVICE
    assert L.parason_kv_read(cache(), rows(), FAKE, FAKE, P.DTYPE_BF16, 1024, 128, None, None) == P.ERR_DEVICE
    assert L.parason_tree_attention(cache(), rows(), tree(), None, FAKE, 1 << 40, None) == P.ERR_DEVICE
    assert L.parason_beam_select(FAKE, 10, 10, P.DTYPE_F32, FAKE, None, 1, 2, FAKE, FAKE, FAKE, FAKE, 1 << 30, None) == P.ERR_DEVICE
    a = (P.BeamArray * 1)(P.BeamArray(FAKE, FAKE + 4096, 16, 16, 16))
    assert L.parason_beam_reorder(FAKE, 4, a, 1, None) == P.ERR_DEVICE


def test_oracle_codes():
    """The oracle's e4m3 rounding against torch's, over every code, every midpoint and random values."""
    torch = pytest.importorskip("torch")
    grid = D.E4M3[:127]
    x = np.concatenate([grid, (grid[1:] + grid[:-1]) / 2, np.random.default_rng(0).uniform(0, 448, 4000),
                        np.exp(np.random.default_rng(1).uniform(-12, 6, 4000))]).astype(np.float32)
    x = np.concatenate([x, -x])
    t = torch.from_numpy(x).to(torch.float8_e4m3fn)
    assert np.array_equal(D.fp8_codes(x.astype(np.float64)), t.view(torch.uint8).numpy())
    every = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).float().numpy()
    assert np.array_equal(D.E4M3.astype(np.float32), every, equal_nan=True)


def test_oracle_attention_against_a_plain_softmax():
    """The oracle's rows, heads and masks against a dense softmax written out for one small case."""
    rng = np.random.default_rng(0)
    q, k, v = rng.standard_normal((3, 4, 16)), rng.standard_normal((7, 2, 16)), rng.standard_normal((7, 2, 16))
    mask = np.array([[0b001], [0b011], [0b101]], np.uint64)
    seen = D.visible(7, 3, 3, mask)
    assert seen.tolist() == [[True] * 5 + [False] * 2, [True] * 6 + [False], [True] * 5 + [False, True]]
    assert D.visible(4, 2).tolist() == [[True, True, True, False], [True] * 4]
    out, lse, _, _ = D.attention(q, k, v, seen, 0.3, 7, 7)
    for i in range(3):
        for h in range(4):
            e = np.array([np.exp(0.3 * np.dot(q[i, h], k[p, h // 2])) if seen[i, p] else 0.0 for p in range(7)])
            assert np.allclose(out[i, h], (e[:, None] * v[:, h // 2]).sum(0) / e.sum(), rtol=1e-12)
            assert np.isclose(lse[i, h], np.log(e.sum()))
