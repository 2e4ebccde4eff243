"""What the backward pass of the rotation leaves out: padding, and heads whose squares float32 does not hold."""
import pytest

from gpu_util import log
from paper_2608_24658_amd import parason as PX

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def dev():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    return torch.device("cuda:0")


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("bad", [float("inf"), float("nan")])
def test_padding_has_no_gradient_whatever_the_weights_are(dev, dtype, bad):
    """Results and gradients of padding are zero where a weight is not finite; other tokens' are as the weight makes them."""
    log("case padding, a weight of %s" % bad)
    x = torch.randn(4, 3, 64, device=dev).to(dtype)
    at = torch.tensor([5, -1, 0, -(2 ** 31)], dtype=torch.int32, device=dev)
    f = torch.rand(32, device=dev, dtype=torch.float64)
    w = torch.ones(64, device=dev, dtype=dtype)
    plain = PX.qk_norm_rotate_grad(x, x, x, x, at, f, q_weight=w, k_weight=w)
    w[[3, 40]] = bad
    for y in PX.qk_norm_rotate(x, x, at, f, q_weight=w, k_weight=w):
        assert (y[[1, 3]] == 0).all() and not torch.isfinite(y[[0, 2]]).all()
    got = PX.qk_norm_rotate_grad(x, x, x, x, at, f, q_weight=w, k_weight=w)
    for name in "qk":
        assert (got[name][[1, 3]] == 0).all() and not torch.isfinite(got[name][[0, 2]]).all()
        assert torch.equal(got[name + "_weight"], plain[name + "_weight"])


@pytest.mark.parametrize("size", [1.0, 1e12, 1e30])
def test_heads_whose_squares_are_infinite_have_no_gradient(dev, size):
    """Their results are zero, and so are the gradients, also where a gradient times a value is beyond float32; the heads
    beside them have theirs."""
    log("case squares beyond float32, gradients of %g" % size)
    x, dy = torch.randn(2, 3, 5, 64, device=dev).unbind()
    dy = dy * size
    at, f = torch.arange(3, dtype=torch.int32, device=dev), torch.rand(32, device=dev, dtype=torch.float64)
    want = PX.qk_norm_rotate_grad(dy, dy, x, x, at, f)
    y = x.clone()
    y[1, 2] = torch.where(x[1, 2] < 0, -1e30, 1e30)
    assert (PX.qk_norm_rotate(y, y, at, f)[0][1, 2] == 0).all()
    got = PX.qk_norm_rotate_grad(dy, dy, y, y, at, f)
    for name in "qk":
        assert (got[name][1, 2] == 0).all() and torch.isfinite(got[name + "_weight"]).all()
        want[name][1, 2] = 0
        assert torch.equal(got[name], want[name])
