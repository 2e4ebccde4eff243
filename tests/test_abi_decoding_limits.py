"""Sizes that a launch cannot take and results that lie over their sources: refused by the host checks, before any HIP
call (the fake pointers are never dereferenced)."""
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
    assert L.parason_beam_reorder(FAKE << 32, MOST + 1, arr(16), 1, None) == P.ERR_SIZE
    assert L.parason_beam_reorder(FAKE << 32, MOST // 2 + 1, arr(16385), 1, None) == P.ERR_SIZE


@no_gpu
def test_as_many_blocks_as_a_launch_takes():
    L = P.lib()
    for fn in (L.parason_kv_write, L.parason_kv_read):
        assert fn(cache(), rows(n_rows=MOST), FAKE, FAKE, P.DTYPE_BF16, 1024, 128, None, None) == P.ERR_DEVICE
    arr = (P.BeamArray * 1)(P.BeamArray(FAKE, FAKE + (1 << 50), 16, 16, 16))
    assert L.parason_beam_reorder(FAKE << 32, MOST, arr, 1, None) == P.ERR_DEVICE
    assert L.parason_beam_select(FAKE, 10, 10, P.DTYPE_F32, FAKE, None, MOST, 1, FAKE, FAKE, FAKE, FAKE, 1 << 40, None) == P.ERR_DEVICE


def test_reorder_over_its_sources():
    fn = P.lib().parason_beam_reorder
    call = lambda *a, n=4, parents=FAKE << 20: fn(parents, n, (P.BeamArray * len(a))(*(P.BeamArray(*x) for x in a)), len(a), None)  # noqa: E731
    far = FAKE << 8
    assert call((FAKE, FAKE, 16, 16, 16)) == P.ERR_PARAM
    assert call((FAKE, FAKE + 48, 16, 16, 16)) == P.ERR_PARAM
    assert call((FAKE + 63, FAKE, 16, 16, 16)) == P.ERR_PARAM
    assert call((FAKE, FAKE + 8, 16, 32, 32)) == P.ERR_PARAM          # rows beside each other, but not quite
    assert call((FAKE, FAKE + 100, 16, 32, 48)) == P.ERR_PARAM        # different strides
    assert call((FAKE, far, 16, 16, 16), (far + 4096, FAKE + 8, 16, 16, 16)) == P.ERR_PARAM   # another array's source
    assert call((FAKE, far, 16, 16, 16), (FAKE, far + 60, 16, 16, 16)) == P.ERR_PARAM         # another array's result
    assert call((FAKE, far, 16, 16, 16), parents=far + 32) == P.ERR_PARAM                     # the parents
    assert call((FAKE, FAKE, 0, 16, 16)) == P.OK                      # nothing to move
    assert call((FAKE, FAKE + 8, 2000, 4000, 4000), n=1 << 20) == P.ERR_PARAM


@no_gpu
def test_reorder_beside_its_sources():
    fn = P.lib().parason_beam_reorder
    call = lambda *a, n=4, parents=FAKE << 20: fn(parents, n, (P.BeamArray * len(a))(*(P.BeamArray(*x) for x in a)), len(a), None)  # noqa: E731
    far = FAKE << 8
    assert call((FAKE, FAKE + 64, 16, 16, 16)) == P.ERR_DEVICE
    assert call((FAKE, FAKE + 16, 16, 32, 32)) == P.ERR_DEVICE        # two columns of one array
    assert call((FAKE + 16, FAKE, 16, 32, 32)) == P.ERR_DEVICE
    assert call((FAKE, FAKE + 16, 16, 64, 32)) == P.ERR_DEVICE        # different strides, rows that miss each other
    assert call((FAKE, far, 16, 16, 16), (FAKE, far + 64, 16, 16, 16)) == P.ERR_DEVICE        # one source twice
    assert call((FAKE, FAKE + 2000, 2000, 4000, 4000), n=1 << 20) == P.ERR_DEVICE
    assert call((FAKE, far, 16, 16, 16), parents=FAKE) == P.ERR_DEVICE                        # the parents moved too
