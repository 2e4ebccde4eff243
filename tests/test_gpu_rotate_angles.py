"""Angles of far positions: the sines and cosines that qk_norm_rotate turns by, against angles that are reduced to a turn in
whole numbers."""
from fractions import Fraction

import numpy as np
import pytest

from gpu_util import log
from paper_2608_24658_amd import parason as PX

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

PI = Fraction("3.14159265358979323846264338327950288419716939937510582097494459")


def reduced(position, freq):
    """position * freq less a whole number of turns, exact but for the last rounding."""
    x = Fraction(int(position)) * Fraction(float(freq))
    return float(x - 2 * PI * round(x / (2 * PI)))


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("low,high", [(0, 100), (50_000, 1 << 20), (1 << 30, 1 << 31)])
def test_angles_are_exact_wherever_the_token_is(low, high, interleaved):
    """Heads with one pair of (4 sqrt 2, 0) among zeros, 32 values whose root mean square is 1: results are 4 sqrt 2 times a
    cosine and a sine.  In units u = 2^-24: 1 / root 3 u, the product with it 1 u, a cosine or sine 4 u and its correction
    2 u, the products by it 2 u, the result 1 u: 13 u of the size in all, wherever the token is.  (An angle of 2^31 that is a
    rounded product of doubles is off by 2^-22 radians, 4 u, and one of 2^34 by 32 u.)"""
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    log("case angles from %d, interleaved %s" % (low, interleaved))
    dev, dim, n = torch.device("cuda:0"), 32, 400
    rng = np.random.default_rng(low)
    at = rng.integers(low, high, n)
    at[:2] = low, high - 1
    freqs = np.array([1.0, 1 / 3, 0.7, 2.0 ** -20, 1e-9, 3.0, 7.9, 6.283185307179586, 0.1, 5.5, 1.0 + 2.0 ** -50, 4.7, 2.2, 0.0, 1e-3, 6.9])
    pairs = np.arange(dim // 2)
    a, b = (2 * pairs, 2 * pairs + 1) if interleaved else (pairs, pairs + dim // 2)
    want = np.zeros((n, dim // 2, dim))
    x = np.zeros((n, dim // 2, dim), np.float32)
    for one in range(dim // 2):
        x[:, one, a[one]] = 4 * np.sqrt(2.0)
        angle = np.array([reduced(p, freqs[one]) for p in at])
        want[:, one, a[one]], want[:, one, b[one]] = np.cos(angle), np.sin(angle)
    size = float(np.float32(4 * np.sqrt(2.0)))
    want *= size / np.sqrt(size * size / dim + 1e-30)
    d = lambda v, t: torch.as_tensor(v).to(device=dev, dtype=t)  # noqa: E731
    q = d(x, torch.float32)
    got, k = PX.qk_norm_rotate(q, q[:, :1], d(at, torch.int32), d(freqs, torch.float64), eps=1e-30, interleaved=interleaved)
    far = np.abs(got.cpu().double().numpy() - want).max()
    log("  within %.1f u" % (far / size * 2.0 ** 24))
    assert far <= 13 * 2.0 ** -24 * size
    assert torch.equal(k[:, 0], got[:, 0])
    # the backward pass turns back by the same angles, and with x = 0 that is all it does: another 8 u of each of two values
    zero = torch.zeros_like(q)
    g = PX.qk_norm_rotate_grad(got, k, zero, zero[:, :1], d(at, torch.int32), d(freqs, torch.float64), eps=1.0, interleaved=interleaved)
    back = g["q"].cpu().double().numpy()
    there = np.zeros_like(want)
    there[:, pairs, a] = np.linalg.norm(want, axis=-1)
    assert np.abs(back - there).max() <= 2 * 13 * 2.0 ** -24 * size
