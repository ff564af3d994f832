"""Layer norm, forward and backward, of rows whose mean is far above their
spread: constant rows of values that use the whole mantissa, and rows of a
common offset.

Bounds, u = 2^-24.  A row's mean is off by at most 16 u max |h| (a sum of few
levels); the mean of the centred values is taken out as well, which leaves 16 u
of that and 16 u of the largest centred value.  So with V = max |h - mean| /
sigma and H = max |h| / sigma the normalised values are off by 64 u (|n| + V +
64 u H), as in the other layer norm tests with V in the place of H, and so on
through the gradients."""
import numpy as np
import pytest

from oracle import routing_oracle as R

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

U = 2.0 ** -24
HALF = {torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}


@pytest.fixture(scope="module", autouse=True)
def _need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2411_01433_amd as P
    P.lib()
    yield


def _f64(t):
    return t.double().cpu().numpy()


def _rows(d, kind, seed):
    """40 rows: constant ones from 10 to 2e4, or a spread of 0.01 on an offset
    of 100 to 200, or a spread of a few steps of fp32."""
    g = torch.Generator().manual_seed(seed)
    u = torch.rand((40, 1), generator=g)
    if kind == "constant":
        h = (1 + u) * 10.0 ** (1 + torch.arange(40) % 4).float()[:, None] * torch.ones((1, d))
    elif kind == "offset":
        h = 100 * (1 + u) + 0.01 * torch.randn((40, d), generator=g)
    else:
        h = 1e6 * (1 + u) + torch.randint(-1, 2, (40, d), generator=g) * (torch.rand((40, d), generator=g) < 0.1)
    return h.cuda(), g


def _spread(h, eps):
    """(|n|, V + 64 u H, 1 / sigma) of rows."""
    c = h - h.mean(-1, keepdims=True)
    r = 1.0 / np.sqrt((c * c).mean(-1, keepdims=True) + eps)
    top = lambda v: np.abs(v).max(-1, keepdims=True) * r
    return np.abs(c * r), top(c) + 64 * U * top(h), r


SIZES = [64, 320, 1088, 4096, 4160, 5120, 16384]


@pytest.mark.parametrize("kind", ["constant", "offset", "steps"])
@pytest.mark.parametrize("d", SIZES)
@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16], ids=["f16", "bf16"])
def test_forward(d, kind, dtype):
    import paper_2411_01433_amd as P
    h, g = _rows(d, kind, d)
    x = torch.empty(h.shape, dtype=dtype, device="cuda")
    for eps in (1e-5, 1e-3):
        P.layernorm(h, x, eps=eps)
        ref = R.layernorm(_f64(h), eps=eps)
        n, V, _ = _spread(_f64(h), eps)
        tol = HALF[dtype] * np.abs(ref) + 64 * U * (n + V) + 2.0 ** -25
        off = np.abs(_f64(x) - ref)
        assert (off <= tol).all(), (eps, off.max(), (off / tol).max())


@pytest.mark.parametrize("kind", ["constant", "offset", "steps"])
@pytest.mark.parametrize("d", SIZES)
def test_backward(d, kind):
    import paper_2411_01433_amd as P
    h, g = _rows(d, kind, d + 1)
    T = h.shape[0]
    gain = (1 + 0.3 * torch.randn(d, generator=g)).cuda()
    dx = torch.randn((T, d), generator=g).half().cuda()
    dh, dg, db = torch.empty_like(h), torch.empty(d, device="cuda"), torch.empty(d, device="cuda")
    eps = 1e-5
    P.layernorm_backward(dx, h, dh, gain, dg, db, eps)
    rh, rg, rb = R.layernorm_backward(_f64(dx), _f64(h), _f64(gain), eps)
    n, V, r = _spread(_f64(h), eps)
    a, m = np.abs(_f64(dx)) * np.abs(_f64(gain)), lambda v: v.mean(-1, keepdims=True)
    tol = 64 * U * r * (a + m(a) + (n + V) * m(a * (n + V)))
    off = np.abs(_f64(dh) - rh)
    assert (off <= tol).all(), ("d_h", (off / tol).max())
    # (as in the other tests: 40 rows, a block each, and the blocks' join)
    off = np.abs(_f64(dg) - rg)
    tol = 96 * U * (np.abs(_f64(dx)) * (n + V)).sum(0)
    assert (off <= tol).all(), ("d_gain", (off / tol).max())
    assert (np.abs(_f64(db) - rb) <= 96 * U * np.abs(_f64(dx)).sum(0)).all()


def test_small_eps_keeps_a_small_spread():
    """A spread of one step of fp32 in a few places, which no epsilon covers."""
    import paper_2411_01433_amd as P
    h, _ = _rows(4160, "steps", 3)
    x = torch.empty(h.shape, dtype=torch.float16, device="cuda")
    P.layernorm(h, x, eps=1e-12)
    ref = R.layernorm(_f64(h), eps=1e-12)
    n, V, _ = _spread(_f64(h), 1e-12)
    off = np.abs(_f64(x) - ref)
    assert (off <= 2.0 ** -11 * np.abs(ref) + 64 * U * (n + V) + 2.0 ** -25).all(), off.max()
