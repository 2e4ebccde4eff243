"""Sizes that a launch cannot take: refused by the host checks, before any HIP call (the fake pointers are never
dereferenced)."""
import ctypes

import pytest

from paper_2608_24658_amd import parason as P
from test_abi_decoding import FAKE, _gpu_visible, cache, rows

MOST = (2 ** 32 - 1) // 256  # blocks of 256 threads
no_gpu = pytest.mark.skipif(_gpu_visible(), reason="with a GPU these calls would pass the device check and launch")


def test_more_blocks_than_a_launch_takes():
    L, ws = P.lib(), ctypes.c_size_t()
    size = L.parason_beam_workspace_size
    assert size(MOST, 1, 10, ctypes.byref(ws)) == P.OK
    assert size(MOST + 1, 1, 10, ctypes.byref(ws)) == P.ERR_SIZE
    assert size(MOST // 64 + 1, 64, 10, ctypes.byref(ws)) == P.ERR_SIZE
    assert size(MOST // 2 + 1, 1, 10000, ctypes.byref(ws)) == P.ERR_SIZE
    assert L.parason_beam_select(FAKE, 10, 10, P.DTYPE_F32, FAKE, None, MOST + 1, 1, FAKE, FAKE, FAKE, FAKE, 1 << 40, None) == P.ERR_SIZE
    for fn in (L.parason_kv_write, L.parason_kv_read):
        assert fn(cache(), rows(n_rows=MOST + 1), FAKE, FAKE, P.DTYPE_BF16, 1024, 128, None, None) == P.ERR_SIZE
    arr = lambda n: (P.BeamArray * 1)(P.BeamArray(FAKE, FAKE + (1 << 50), n, n, n))  # noqa: E731
    assert L.parason_beam_reorder(FAKE << 30, MOST + 1, arr(16), 1, None) == P.ERR_SIZE
    assert L.parason_beam_reorder(FAKE << 30, MOST // 2 + 1, arr(16385), 1, None) == P.ERR_SIZE


@no_gpu
def test_as_many_blocks_as_a_launch_takes():
    L = P.lib()
    for fn in (L.parason_kv_write, L.parason_kv_read):
        assert fn(cache(), rows(n_rows=MOST), FAKE, FAKE, P.DTYPE_BF16, 1024, 128, None, None) == P.ERR_DEVICE
    arr = (P.BeamArray * 1)(P.BeamArray(FAKE, FAKE + (1 << 50), 16, 16, 16))
    assert L.parason_beam_reorder(FAKE << 30, MOST, arr, 1, None) == P.ERR_DEVICE
    assert L.parason_beam_select(FAKE, 10, 10, P.DTYPE_F32, FAKE, None, MOST, 1, FAKE, FAKE, FAKE, FAKE, 1 << 40, None) == P.ERR_DEVICE
