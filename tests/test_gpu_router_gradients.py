"""Bits that the routing's gradients hold, at inputs where they show.

Where a token has a gradient for one expert alone, d_x is one product and
d_w_router a sum of as many products as tokens have that expert: the exact
values are known, and what is off is the rounding of the logits' gradient into
parts of 16 bits (fp16 two: 2^-23 of a value; bf16 three: 2^-25), of the sums
and of the output.  A step of the matrix cores cuts each of its products at
2^-24 of its largest, cuts the sum so far there and rounds it: with n products
in a sum of one part at most 3 n of 2^-24."""
import numpy as np
import pytest

from oracle import routing_oracle as R
from test_gpu_router import BF16, F16, U, _np, make

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.fixture(scope="module", autouse=True)
def _need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2411_01433_amd as P
    P.lib()
    yield


def half_step(v, dtype):
    """Half a step of `dtype` at the values v, subnormals among them."""
    bits, least = (11, -14) if dtype is F16 else (8, -126)
    e = np.maximum(np.floor(np.log2(np.maximum(np.abs(v), 1e-300))), least)
    return 2.0 ** (e - bits)


def one_expert_each(T, d, E, dtype, seed):
    """x, gate, a gradient of the logits with one expert per token, its experts."""
    g = torch.Generator().manual_seed(seed)
    x = torch.randn((T, d), generator=g).to(dtype).cuda()
    wg = torch.randn((E, d), generator=g).to(dtype).cuda()
    e = torch.arange(T) % E
    v = torch.randn(T, generator=g)
    dl = torch.zeros((T, E))
    dl[torch.arange(T), e] = v
    return x, wg, dl, e


def backward(x, wg, dl, rule=R.Rule(1)):
    """(d_x, d_w_router) from a gradient of the logits alone."""
    T, E = dl.shape
    r = make(rule, wg, None, T, backward=True)
    dx, dw = torch.empty_like(x), torch.empty(wg.shape, device="cuda")
    idx = torch.full((T, rule.top_k), -1, dtype=torch.int32, device="cuda")
    r.backward(x, torch.zeros((T, E), device="cuda"), idx,
               torch.zeros((T, rule.top_k), device="cuda"), dx, dw, dl.cuda())
    torch.cuda.synchronize()
    r.destroy()
    return _np(dx), _np(dw)


@pytest.mark.parametrize("dtype", [F16, BF16], ids=["f16", "bf16"])
@pytest.mark.parametrize("T,d,E", [(64, 1024, 5), (130, 320, 60), (300, 256, 160), (100, 192, 512)])
def test_products_hold_their_bits(T, d, E, dtype):
    """d_x: the product of three parts at most, 9 + 1 of 2^-24, rounded once to
    the output's type.  d_w_router: n tokens of an expert in 64, whose sums are
    added (twice 2^-24 each, scale and sum)."""
    x, wg, dl, e = one_expert_each(T, d, E, dtype, T + E)
    dx, dw = backward(x, wg, dl)
    want = dl.double().numpy() @ _np(wg)
    off = np.abs(dx - want)
    tol = half_step(want, dtype) + 11 * U * np.abs(want)
    assert (off <= tol).all(), ((off > tol).mean(), (off / tol).max())
    want = dl.double().numpy().T @ _np(x)
    of = np.abs(dl.double().numpy()).T @ np.abs(_np(x))
    n, sets = -(-64 // E), -(-T // 64)
    assert (np.abs(dw - want) <= (9 * n + 2 + 2 * sets) * U * of).all()


@pytest.mark.parametrize("dtype", [F16, BF16], ids=["f16", "bf16"])
@pytest.mark.parametrize("T,d,E", [(64, 256, 64), (192, 128, 160), (70, 320, 24)])
def test_small_gradients_beside_large_ones(T, d, E, dtype):
    """Experts whose gradients are 2^-6 to 2^-60 of others' in the same tokens
    keep the bits of their gate rows, and tokens beside one whose gradient is
    2^60 times theirs (and leaves the range of fp16) the bits of their d_x."""
    x, wg, dl, e = one_expert_each(T, d, E, dtype, 5 * T)
    for step in (6, 12):
        small = dl * torch.exp2(-step * (torch.arange(E) % 6).float())
        _, dw = backward(x, wg, small)
        want = small.double().numpy().T @ _np(x)
        of = np.abs(small.double().numpy()).T @ np.abs(_np(x))
        n, sets = -(-64 // E), -(-T // 64)
        assert (np.abs(dw - want) <= (9 * n + 2 + 2 * sets) * U * of).all()
    dl[3] *= 2.0 ** 60
    dx, _ = backward(x, wg, dl)
    want = dl.double().numpy() @ _np(wg)
    rest = np.arange(T) != 3
    tol = half_step(want, dtype) + 11 * U * np.abs(want)
    assert (np.abs(dx - want) <= tol)[rest].all()
    if dtype is F16:
        far = np.abs(want[3]) > 2 * 65504
        assert far.any() and np.isinf(dx[3, far]).all()


def test_unlikely_experts_of_a_softmax_over_all():
    """Gate rows of experts whose logits lie 15, 20 and 25 below the rest, whose
    gradients are products of their scores: within the functions' rounding, 64 u
    (1 + the largest |logit|) of every term, the parts' and the sums'."""
    T, d, E = 128, 192, 60
    rule = R.Rule(4, renormalize=False)
    g = torch.Generator().manual_seed(3)
    x = torch.randn((T, d), generator=g).half().cuda()
    wg = (torch.randn((E, d), generator=g) * 0.05).half().cuda()
    l = x.float() @ wg.float().T
    l[:, 7] -= 15
    l[:, 8] -= 20
    l[:, 9] -= 25
    l64 = _np(l)
    idx = np.stack([R.select(rule, r) for r in l64])
    dw = torch.randn((T, 4), generator=g)
    r = make(rule, wg, None, T, backward=True)
    out = torch.empty((E, d), device="cuda")
    r.backward(x, l, torch.from_numpy(idx).cuda(), dw.cuda(), None, out)
    torch.cuda.synchronize()
    r.destroy()
    _, want, _ = R.route_backward(rule, _np(x), _np(wg), l64, idx, dw.numpy())
    # magnitudes of the terms: the softmax's mean is a sum of four
    terms = np.stack([R.scores(rule, l64[t]) * (np.abs(dw[t].numpy() * R.scores(rule, l64[t])[idx[t]]).sum()
                      + np.isin(np.arange(E), idx[t]) * np.abs(dw[t].numpy()).max()) for t in range(T)])
    of = terms.T @ np.abs(_np(x))
    # (64 tokens in each of two parts: 3 x 64 x 2 of 2^-24, and the functions')
    big = 1 + np.abs(l64).max()
    assert (np.abs(_np(out) - want) <= (64 * big + 3 * 128 + 6) * U * of).all()


@pytest.mark.parametrize("dtype", [F16, BF16], ids=["f16", "bf16"])
@pytest.mark.parametrize("T,E", [(70, 8), (150, 60), (200, 100), (321, 256)])
def test_tokens_without_a_gradient_may_hold_anything(T, E, dtype):
    """Padded rows of NaN and infinities, whose slots are empty or whose
    gradients are zero, among the others: the gradients of a call in which
    those rows are zeros, bit for bit."""
    d, rule = 192, R.Rule(4, score=R.SIGMOID)
    g = torch.Generator().manual_seed(T)
    x = torch.randn((T, d), generator=g).to(dtype)
    wg = (torch.randn((E, d), generator=g) * 0.1).to(dtype).cuda()
    pad = torch.zeros(T, dtype=torch.bool)
    pad[3:9] = pad[63:65] = pad[T - 5:] = True
    if T > 192:
        pad[128:192] = True   # 64 tokens that the kernels take together
    clean = torch.where(pad[:, None], torch.zeros_like(x), x).cuda()
    x[pad] = float("nan")
    x[4], x[7, :9] = float("inf"), -float("inf")
    x = x.cuda()
    r = make(rule, wg, None, T, backward=True)
    idx = torch.empty((T, 4), dtype=torch.int32, device="cuda")
    w, lg = torch.empty((T, 4), device="cuda"), torch.empty((T, E), device="cuda")
    r.route(x, idx, w, lg)
    assert (idx[pad.cuda()] == -1).all()
    up = torch.randn((T, 4), generator=g).cuda()
    dl = (0.1 * torch.randn((T, E), generator=g))
    dl[pad] = 0
    for extra in (None, dl.cuda()):
        got, want = [], []
        for v, into in ((x, got), (clean, want)):
            dx, dw = torch.empty_like(x), torch.empty((E, d), device="cuda")
            r.backward(v, lg, idx, up, dx, dw, extra)
            into += [dx, dw]
        assert torch.isfinite(want[1]).all() and (want[0][pad.cuda()] == 0).all()
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    r.destroy()
