"""What a serving step leaves in a 4-bit cache: the codes and scales of the keys that it turned, bit for bit, where the tables
say."""
import numpy as np
import pytest

from gpu_util import log
from oracle import serving_oracle as S
from test_gpu_serving_step import DIM, GROUP, HEADS, PAGE, Engine, dev  # noqa: F401

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


def test_the_cache_holds_what_the_steps_wrote(dev):  # noqa: F811
    log("case codes of serving steps")
    rng = np.random.default_rng(2)
    rows, n_pages, q_heads = 4, 50, HEADS * GROUP
    E = Engine(dev, rows, n_pages)
    raw = lambda: [t.view(torch.uint8).cpu().numpy() for t in E.cache]  # noqa: E731
    expect = [t.copy() for t in raw()]
    for n_step in range(4):
        lengths = rng.integers(1, 30, rows) if n_step == 0 else (rng.random(rows) < 0.7).astype(np.int64)
        x = torch.randn(int(lengths.sum()) + 2, q_heads + 2 * HEADS, DIM, device=dev).bfloat16()
        _, at = E.step(x, torch.as_tensor(lengths).to(device=dev, dtype=torch.int32), 30, 200)
        slots = at["slots"].cpu().numpy()
        y = x.float().cpu().numpy()  # keys turned in place, and values
        for t in np.nonzero(slots >= 0)[0]:
            page, slot = divmod(int(slots[t]), PAGE)
            for w, first in enumerate((q_heads, q_heads + HEADS)):
                codes, scales = S.quantise4(y[t, first: first + HEADS])
                expect[w][page, slot], expect[2 + w][page, slot] = S.pack4(codes), scales
        assert int((slots >= 0).sum()) == int(lengths.sum())
        for name, g, want in zip(("k", "v", "k_scale", "v_scale"), raw(), expect):
            assert np.array_equal(g, want), (n_step, name)
