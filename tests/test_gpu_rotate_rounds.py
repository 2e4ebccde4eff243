"""The backward pass of norm and rotation over more tokens than its blocks take in one round (1,024 blocks of at most 16
tokens, or as many as 1,024 angles serve): angles of the second round, weights' gradients carried over it."""
import numpy as np
import pytest

from gpu_util import log
from oracle import serving_oracle as S
from paper_2608_24658_amd import parason as PX
from test_gpu_rotate import dev, make, near, numbers  # noqa: F401

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("given", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("n,q_heads,k_heads,dim,turned", [(33001, 4, 1, 64, 64), (17000, 1, 1, 32, 0), (9001, 2, 1, 256, 256)])
def test_several_rounds(dev, n, q_heads, k_heads, dim, turned, given, interleaved):  # noqa: F811
    log("case rotate back %d tokens dim %d %s %s" % (n, dim, given, interleaved))
    assert n > 1024 * min(16, 2048 // turned if turned else 16)
    q, k, w, at, freqs, qd, kd, call = make(dev, given, n, q_heads, k_heads, dim, turned, seed=n)
    dy = torch.as_tensor(numbers(np.random.default_rng(n), n, q_heads + k_heads, dim).astype(np.float32)).to(qd.dtype)
    dq, dk = dy[:, :q_heads], dy[:, q_heads:]
    got = PX.qk_norm_rotate_grad(dq.to(dev), dk.to(dev), qd, kd, interleaved=interleaved, eps=1e-5, **call)
    for name, x, d, weight in (("q", q, dq, w[0]), ("k", k, dk, w[1])):
        dx, dw, dx_tol, dw_tol = S.rotate_grad(x, d.double().numpy(), weight, at, freqs, 1e-5, interleaved)
        near(got[name], dx, dx_tol, given, "d" + name)
        # the oracle's bound grows with the terms; it says something here because a round left out or counted twice would
        # change the sum by about its share's root
        far = np.abs(got[name + "_weight"].cpu().double().numpy() - dw)
        assert np.all(far <= dw_tol), (name, (far / dw_tol).max())
    # whole numbers, whose sums are exact: x of ones, no rotation, a gradient of 1 for every third token
    one = torch.ones(n, q_heads + k_heads, dim, device=dev)
    g = (torch.arange(n, device=dev) % 3 == 0).float()[:, None, None] * one
    flat = torch.zeros(turned // 2, dtype=torch.float64, device=dev)
    zero = torch.zeros(n, dtype=torch.int32, device=dev)
    got = PX.qk_norm_rotate_grad(g[:, :q_heads], g[:, q_heads:], one[:, :q_heads], one[:, q_heads:], zero, flat, eps=1e-30,
                                 interleaved=interleaved)
    for name, heads in (("q", q_heads), ("k", k_heads)):
        # 1 / root is off by 3 u at most, whichever way, the same for every token: its sums (below 2^24 terms) by 3 u and
        # their own roundings, one a term of a lane's: some hundreds, over the blocks in double
        want = heads * ((n + 2) // 3)
        assert np.abs(got[name + "_weight"].cpu().double().numpy() / want - 1).max() < 0.4 / want
