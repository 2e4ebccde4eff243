"""Reads of many tokens from a 4-bit cache, eight heads at a time, in every type and at every alignment."""
import pytest

from decoding_cases import torch_type
from gpu_util import log
from oracle import serving_oracle as S
from paper_2608_24658_amd import parason as PX
from test_gpu_kv4 import dev  # noqa: F401

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("heads,dim,odd", [(5, 96, False), (5, 32, True), (8, 32, False), (11, 192, False), (11, 96, True)])
@pytest.mark.parametrize("to", ["fp32", "fp16", "bf16"])
def test_many_tokens_of_many_heads(dev, to, heads, dim, odd):  # noqa: F811
    """The last of the heads that are read together are not there; heads of 96 and 192 values are not a power of two of
    lanes, and half of 32 or 96 is not a whole number of scales.  odd: results at 4 or 2 bytes' alignment, around which
    nothing is written.  The first and last tokens, and every thirteenth between them, are compared."""
    log("case kv4 reads to %s, %d heads of %d, odd %s" % (to, heads, dim, odd))
    n = 16400
    cache = PX.kv_alloc(-(-n // 16) + 1, 16, heads, dim, torch.float4_e2m1fn_x2, dev)
    one = lambda v, dt: torch.tensor([v], dtype=dt, device=dev)  # noqa: E731
    pages = torch.randperm(cache.k.shape[0], device=dev, dtype=torch.int32)[None]
    rows = PX.KVRows(one(0, torch.int64), one(n, torch.int32), one(n, torch.int32), pages, n, n)
    # scales of a head lie far apart, and some of its 32s are NaN
    x = torch.randn(2, n, heads, dim // 32, 32, device=dev) * 2.0 ** torch.randint(-6, 7, (2, n, heads, dim // 32, 1), device=dev)
    x[:, ::91, heads - 1, 0, 3] = float("nan")
    x = x.view(2, n, heads, dim)
    PX.kv_write(x[0], x[1], cache, rows)
    wide = torch.full((2, n, heads + 1, dim + (3 if odd else 0)), 5.0, device=dev, dtype=torch_type(to))
    at = slice(1, dim + 1) if odd else slice(0, dim)
    k, v = PX.kv_read(cache, rows, n, wide.dtype, out=(wide[0, :, :heads, at], wide[1, :, :heads, at]))
    t = torch.arange(n)
    t = t[(t < 300) | (t >= n - 300) | (t % 13 == 0)].to(dev)
    for g, w in ((k[t], x[0, t]), (v[t], x[1, t])):
        want = torch.from_numpy(S.values4(*S.quantise4(w.cpu().numpy()))).to(wide.dtype)
        assert torch.equal(torch.nan_to_num(g.cpu().float(), nan=12345.0), torch.nan_to_num(want.float(), nan=12345.0))
    assert (wide[:, :, heads] == 5.0).all() and (not odd or ((wide[..., 0] == 5.0).all() and (wide[..., dim + 1:] == 5.0).all()))
