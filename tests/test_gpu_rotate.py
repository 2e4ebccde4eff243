"""Norm and rotation of queries and keys on the GPU, and the backward pass, against the oracle in 64 bits, within the
error bounds that it derives."""
import numpy as np
import pytest

from decoding_cases import torch_type
from gpu_util import log
from oracle import serving_oracle as S
from paper_2608_24658_amd import parason as PX

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def dev():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    return torch.device("cuda:0")


# half an ulp relative to a value, and half the smallest step of a type
HALF = {"fp32": (2.0 ** -24, 2.0 ** -150), "bf16": (2.0 ** -8, 2.0 ** -134), "fp16": (2.0 ** -11, 2.0 ** -25)}


def numbers(rng, n, heads, dim):
    return rng.standard_normal((n, heads, dim)) * np.exp(rng.uniform(-2, 2, (n, heads, 1)))


def make(dev, given, n, q_heads, k_heads, dim, turned, seed, packed=True, far=50000, padding=True, off=0):
    """Views of one packed projection (or tensors of their own), positions and the like; with their 64-bit values."""
    rng = np.random.default_rng(seed)
    dt = torch_type(given)
    x = torch.as_tensor(numbers(rng, n, q_heads + 2 * k_heads, dim).astype(np.float32)).to(dt)
    at = rng.integers(0, far, n)
    if padding and n > 2:
        at[rng.integers(0, n, max(1, n // 10))] = rng.choice([-1, -(2 ** 31)])
    freqs = 1.0 / 1e4 ** (np.arange(turned // 2) / max(1, turned // 2))
    w = torch.as_tensor((1 + 0.5 * rng.standard_normal((2, dim))).astype(np.float32)).to(dt)
    q, k = x[:, :q_heads], x[:, q_heads: q_heads + k_heads]
    if packed:
        wide = torch.zeros(n, q_heads + 2 * k_heads, dim + off, dtype=dt, device=dev)
        wide[..., off:] = x.to(dev)
        qd, kd = wide[:, :q_heads, off:], wide[:, q_heads: q_heads + k_heads, off:]
    else:
        qd, kd = q.clone().to(dev), k.clone().to(dev)
    call = dict(positions=torch.as_tensor(at).to(device=dev, dtype=torch.int32), freqs=torch.as_tensor(freqs).to(dev), q_weight=w[0].to(dev),
                k_weight=w[1].to(dev))
    return q.double().numpy(), k.double().numpy(), w.double().numpy(), at, freqs, qd, kd, call


def near(got, want, tol, given, what):
    rel, least = HALF[given]
    got = got.detach().cpu().double().numpy()
    top = {"fp16": 65504.0}.get(given, 3.3e38)
    far = np.abs(got - want) / (tol + (np.abs(want) + tol) * rel + least)
    fine = np.abs(want) < top
    assert far[fine].max(initial=0) <= 1, (what, np.unravel_index(far.argmax(), far.shape), far.max())
    return far[fine].max(initial=0)


SHAPES = [
    # tokens, query heads, key heads, dim, turned
    (1, 1, 1, 16, 16), (3, 4, 2, 64, 64), (64, 32, 8, 128, 128), (5, 7, 1, 80, 32), (9, 3, 3, 256, 256), (2, 16, 16, 96, 96), (300, 5, 5, 48, 48),
    (4, 2, 1, 192, 64), (33, 6, 2, 112, 0), (2100, 3, 1, 64, 48), (1, 64, 8, 128, 64), (6, 4, 0, 32, 32), (6, 0, 3, 32, 16),
]


@pytest.mark.parametrize("given", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("shape", SHAPES)
def test_forward(dev, given, interleaved, shape):
    n, q_heads, k_heads, dim, turned = shape
    log("case rotate %s %s %s" % (given, interleaved, shape))
    packed = bool((n + dim // 16) % 3)
    q, k, w, at, freqs, qd, kd, call = make(dev, given, n, q_heads, k_heads, dim, turned, seed=dim + n, packed=packed, off=(n % 2) * 3)
    got = PX.qk_norm_rotate(qd, kd, interleaved=interleaved, eps=1e-5, **call)
    for x, weight, g, name in ((q, w[0], got[0], "q"), (k, w[1], got[1], "k")):
        if x.size:
            want, tol = S.rotate(x, weight, at, freqs, 1e-5, interleaved)
            near(g, want, tol, given, name)
    # no weights; in place
    want = PX.qk_norm_rotate(qd, kd, call["positions"], call["freqs"], interleaved=interleaved)
    if q.size:
        near(want[0], *S.rotate(q, None, at, freqs, 1e-6, interleaved), given, "q without weights")
    rest = qd.new_tensor(7.0)
    around = None
    if packed:
        base = qd._base if qd._base is not None else kd._base
        around = base.clone()
    res = PX.qk_norm_rotate(qd, kd, call["positions"], call["freqs"], interleaved=interleaved, out=(qd, kd))
    assert res[0] is qd and torch.equal(qd, want[0]) and torch.equal(kd, want[1]) and float(rest) == 7.0
    if packed:  # nothing else of the projection has changed
        off = (n % 2) * 3
        around[:, :q_heads, off:], around[:, q_heads: q_heads + k_heads, off:] = want
        assert torch.equal(base, around)


@pytest.mark.parametrize("given", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("shape", SHAPES)
def test_backward(dev, given, interleaved, shape):
    n, q_heads, k_heads, dim, turned = shape
    log("case rotate back %s %s %s" % (given, interleaved, shape))
    packed = bool((n + dim // 16) % 3)
    q, k, w, at, freqs, qd, kd, call = make(dev, given, n, q_heads, k_heads, dim, turned, seed=dim + n, packed=packed, off=(n % 2) * 3)
    rng = np.random.default_rng(n)
    g = torch.as_tensor(numbers(rng, n, q_heads + k_heads, dim).astype(np.float32)).to(torch_type(given))
    g[torch.as_tensor(at < 0)] = float("nan")  # padding's gradients mean nothing
    gd = g.to(dev)
    dq, dk = gd[:, :q_heads], gd[:, q_heads:]
    got = PX.qk_norm_rotate_grad(dq, dk, qd, kd, interleaved=interleaved, eps=1e-5, **call)
    again = PX.qk_norm_rotate_grad(dq, dk, qd, kd, interleaved=interleaved, eps=1e-5, **call)
    for name, x, dy, weight in (("q", q, g[:, :q_heads], w[0]), ("k", k, g[:, q_heads:], w[1])):
        dw = got[name + "_weight"]
        assert torch.equal(dw, again[name + "_weight"]) and torch.equal(got[name], again[name])
        if not x.size:
            assert (dw == 0).all()
            continue
        dx, dw_want, dx_tol, dw_tol = S.rotate_grad(x, dy.double().numpy(), weight, at, freqs, 1e-5, interleaved)
        near(got[name], dx, dx_tol, given, "d" + name)
        far = np.abs(dw.cpu().double().numpy() - dw_want) / (dw_tol + 1e-300)
        assert far.max() <= 1, (name, far.max())
    # over the gradients; without the weights'
    res = PX.qk_norm_rotate_grad(dq, dk, qd, kd, interleaved=interleaved, eps=1e-5, out=(dq, dk), weights=False, **call)
    assert sorted(res) == ["k", "q"] and torch.equal(dq, got["q"]) and torch.equal(dk, got["k"])


def test_weight_gradients_of_many_tokens(dev):
    """More tokens than the blocks take at once, ones for x and dy: the weights' gradients are the tokens times the heads
    times 1 / sqrt(1 + eps), every token counted once (one more or less is 3e-5 of it)."""
    log("case many tokens")
    n, dim = 9001, 64
    q, k = torch.ones(n, 4, dim, device=dev), torch.ones(n, 1, dim, device=dev)
    at = torch.zeros(n, dtype=torch.int32, device=dev)
    for turned in (0, 32):
        f = torch.zeros(turned // 2, dtype=torch.float64, device=dev)
        got = PX.qk_norm_rotate_grad(q, k, q, k, at, f, eps=1e-6)
        for name, heads in (("q", 4), ("k", 1)):
            want = n * heads / np.sqrt(1 + 1e-6)
            assert np.abs(got[name + "_weight"].cpu().double().numpy() / want - 1).max() < 1e-5


def test_far_positions(dev):
    """Angles of 2^31 radians are exact to their last bits in float32 results."""
    log("case far positions")
    at = np.array([0, 1, 2 ** 31 - 1, 2 ** 30 + 12345, 777777777, 3])
    x = np.random.default_rng(0).standard_normal((6, 2, 32)).astype(np.float32)
    freqs = np.array([1.0, 0.5, 1e-3, 2.0 ** -20, 1e-9, 0.0, 3.0, 0.7] * 2)
    d = lambda a, t: torch.as_tensor(a).to(device=dev, dtype=t)  # noqa: E731
    got, _ = PX.qk_norm_rotate(d(x, torch.float32), d(x, torch.float32), d(at, torch.int32), d(freqs, torch.float64))
    near(got, *S.rotate(x, None, at, freqs, 1e-6, False), "fp32", "far")


def test_values_that_are_not_finite(dev):
    """A head with a NaN or an infinity is NaN where it says so, its neighbours are whole; zeros stay zeros; squares
    beyond float32 give zeros."""
    log("case not finite")
    x = torch.randn(5, 2, 64, device=dev)
    at, f = torch.arange(5, dtype=torch.int32, device=dev), torch.rand(32, device=dev, dtype=torch.float64)
    want = PX.qk_norm_rotate(x, x, at, f)[0].clone()
    y = x.clone()
    y[1, 0, 3], y[2, 1, 40], y[3, 0], y[4, 1] = float("nan"), float("inf"), 0.0, 1e30
    got = PX.qk_norm_rotate(y, y, at, f)[0]
    assert torch.isnan(got[1, 0]).all() and torch.isnan(got[2, 1, [8, 40]]).all() and (got[3, 0] == 0).all() and (got[4, 1] == 0).all()
    for t, h in ((0, 0), (0, 1), (1, 1), (2, 0), (3, 1), (4, 0)):
        assert torch.equal(got[t, h], want[t, h])
    y[:] = float("nan")
    at[:] = -1
    assert (PX.qk_norm_rotate(y, y, at, f)[0] == 0).all()
    res = PX.qk_norm_rotate_grad(y, y, y, y, at, f)
    assert all((t == 0).all() for t in res.values())


def test_offsets_beyond_32_bits(dev):
    """Tokens whose values lie behind 2^32 of the first one's, in and out."""
    log("case rotation long offsets")
    n, q_heads, k_heads, dim, stride = 4, 3, 2, 64, 1_500_000_016
    q, k, w, at, freqs, _, _, call = make(dev, "bf16", n, q_heads, k_heads, dim, dim, 5, packed=False, padding=False)
    dq, dk = (torch.randn(x.shape, generator=torch.Generator().manual_seed(i)).bfloat16().double().numpy() for i, x in enumerate((q, k)))
    wide = [torch.empty((n - 1) * stride + (q_heads + k_heads) * dim, dtype=torch.bfloat16, device=dev) for _ in range(2)]
    heads = [(b.as_strided((n, q_heads, dim), (stride, dim, 1)), b.as_strided((n, k_heads, dim), (stride, dim, 1), q_heads * dim)) for b in wide]
    for views, values in zip(heads, ((q, k), (dq, dk))):
        for v, x in zip(views, values):
            v.copy_(torch.as_tensor(x))
    grads = PX.qk_norm_rotate_grad(*heads[1], *heads[0], out=heads[1], **call)
    got = PX.qk_norm_rotate(*heads[0], out=heads[0], **call)
    for i, (x, dy, name) in enumerate(((q, dq, "q"), (k, dk, "k"))):
        near(got[i], *S.rotate(x, w[i], at, freqs, 1e-6, False), "bf16", name)
        dx, dw, dx_tol, dw_tol = S.rotate_grad(x, dy, w[i], at, freqs, 1e-6, False)
        near(grads[name], dx, dx_tol, "bf16", "gradient of " + name)
        assert (np.abs(grads[name + "_weight"].cpu().double().numpy() - dw) <= dw_tol).all()


def test_the_smallest_eps(dev):
    """Heads of zeros, and padding, with an eps that is no normal number: zeros, and no gradient that is not finite."""
    log("case smallest eps")
    x, at = torch.zeros(3, 2, 64, device=dev), torch.tensor([0, 5, -1], dtype=torch.int32, device=dev)
    x[2] = float("nan")
    f = torch.rand(32, device=dev, dtype=torch.float64)
    assert all((t == 0).all() for t in PX.qk_norm_rotate(x, x, at, f, eps=1e-44))
    res = PX.qk_norm_rotate_grad(x, x, x, x, at, f, eps=1e-44)
    assert all((t == 0).all() for t in res.values())


def test_no_tokens(dev):
    log("case no tokens")
    x = torch.empty(0, 3, 64, device=dev, dtype=torch.bfloat16)
    at, f = torch.empty(0, dtype=torch.int32, device=dev), torch.rand(32, device=dev, dtype=torch.float64)
    q, k = PX.qk_norm_rotate(x, x[:, :1], at, f)
    assert q.shape == (0, 3, 64) and k.shape == (0, 1, 64)
    res = PX.qk_norm_rotate_grad(x, x[:, :1], x, x[:, :1], at, f)
    assert (res["q_weight"] == 0).all() and (res["k_weight"] == 0).all()


def test_refusals(dev):
    log("case refusals")
    x = torch.randn(4, 3, 64, device=dev, dtype=torch.bfloat16)
    at, f = torch.arange(4, dtype=torch.int32, device=dev), torch.rand(32, device=dev, dtype=torch.float64)
    w = torch.ones(64, device=dev, dtype=torch.bfloat16)
    for args, kw in (((x, x.float(), at, f), {}), ((x.transpose(1, 2), x.transpose(1, 2), at, f), {}), ((x[0], x[0], at, f), {}),
                     ((x, x, at.long(), f), {}), ((x, x, at[:3], f), {}), ((x, x, at, f.float()), {}), ((x, x, at, f[::2]), {}),
                     ((x, x, at, f), dict(q_weight=w.float())), ((x, x, at, f), dict(k_weight=w[:32])), ((x, x[:3], at, f), {}),
                     ((x, x, at, f), dict(out=(x.float(), x))), ((x, x, at, f), dict(out=(x[:, :1], x)))):
        with pytest.raises((TypeError, ValueError)):
            PX.qk_norm_rotate(*args, **kw)
    with pytest.raises(PX.ParasonError):
        PX.qk_norm_rotate(x, x, at, torch.rand(20, device=dev, dtype=torch.float64))
    with pytest.raises(PX.ParasonError):
        PX.qk_norm_rotate(x, x, at, f, eps=0)
    wants = x.clone().requires_grad_()
    with pytest.raises(RuntimeError):
        PX.qk_norm_rotate(wants, x, at, f)
    with torch.no_grad():
        assert torch.equal(PX.qk_norm_rotate(wants, x, at, f)[0], PX.qk_norm_rotate(x, x, at, f)[0])
    for ws in (torch.empty(1 << 20, dtype=torch.uint8), torch.empty(1 << 20, device=dev)):
        with pytest.raises(TypeError):
            PX.qk_norm_rotate_grad(x, x, x, x, at, f, workspace=ws)
    with pytest.raises(PX.ParasonError):
        PX.qk_norm_rotate_grad(x, x, x, x, at, f, workspace=torch.empty(100, dtype=torch.uint8, device=dev))


def test_on_another_stream_and_in_a_graph(dev):
    log("case streams and graphs")
    *_, qd, kd, call = make(dev, "bf16", 1500, 4, 2, 64, 64, seed=1, padding=False)
    dq, dk = torch.randn_like(qd), torch.randn_like(kd)
    want = PX.qk_norm_rotate(qd, kd, **call)
    back = PX.qk_norm_rotate_grad(dq, dk, qd, kd, **call)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        got = PX.qk_norm_rotate(qd, kd, **call)
    s.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        y = PX.qk_norm_rotate(qd, kd, **call)
        d = PX.qk_norm_rotate_grad(dq, dk, qd, kd, **call)
    for _ in range(3):
        for t in tuple(y) + tuple(d.values()):
            t.fill_(5)
        (torch.randn(1000, device=dev) * 2).sum().item()
        g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(y, want)) and all(torch.equal(d[k], back[k]) for k in back)
