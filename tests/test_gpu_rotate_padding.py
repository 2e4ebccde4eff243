"""What the backward pass of the rotation leaves out: padding."""
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
