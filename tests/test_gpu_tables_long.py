"""Rows that give back more pages than one wave takes, in tables that are too large for one block."""
import numpy as np
import pytest

from gpu_util import log
from serving_cases import Tables
from test_gpu_tables import dev  # noqa: F401

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("page", [1, 4])
@pytest.mark.parametrize("rows", [40, 4100])
def test_rows_of_many_pages(dev, rows, page):  # noqa: F811
    """Rows that lose 512 pages, one less and one more, some thousand, and all of theirs, between short ones; the pages come
    off the pool again in the order in which the rows had them."""
    log("case tables of %d rows that lose many pages of %d" % (rows, page))
    rng = np.random.default_rng(rows)
    kv = rng.integers(0, 9 * page, rows)
    long = dict(zip((0, 7, 8, 20, 33, rows - 1), ((1024, 512), (700, 189), (513, 0), (1751, 214), (1537, 1), (2000, 0))))  # pages before, after
    for i, (had, _) in long.items():
        kv[i] = had * page - rng.integers(0, page)
    T = Tables(dev, kv, page, 2001, seed=1, spare=9, pad=page % 3)
    assert rows * 2001 > 64 * 1024
    keeps = np.where(rng.random(rows) < 0.5, kv, kv // 2)
    for i, (_, stay) in long.items():
        keeps[i] = max(0, stay * page - rng.integers(0, page))
    before = [t.clone() for t in (T.d_lens, T.d_pages)]
    T.shrink(keeps)
    T.extend(kv - keeps)
    T.shrink(keeps)
    T.extend(kv - keeps)
    assert torch.equal(T.d_lens, before[0]) and torch.equal(T.d_pages, before[1])
    T.shrink(np.zeros(rows))
    assert T.count == T.free.size and (T.pages == -1).all()
