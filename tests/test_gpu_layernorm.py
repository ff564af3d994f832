"""Layer norm and its backward pass against the float64 oracle.

Bounds.  u = 2^-24 is half a step of fp32, H = max |h| / sigma of a row.  A
normalised value n carries the rounding of the mean (of numbers up to H, sums
of a few levels) and of the centring: 32 u (|n| + H) covers both, and the
scale's 32 u |n|.  An output of 16 bits adds half a step of its type (and half
of the smallest subnormal of fp16)."""
import numpy as np
import pytest

from oracle import routing_oracle as R

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

U = 2.0 ** -24
HALF = {torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}
EPS = 1e-5


@pytest.fixture(scope="module", autouse=True)
def _need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2411_01433_amd as P
    P.lib()
    yield


def _f64(t):
    return t.double().cpu().numpy()


def _rows(T, d, seed, offset=0.5):
    g = torch.Generator().manual_seed(seed)
    h = torch.randn((T, d), generator=g) + offset * torch.randn((T, 1), generator=g)
    h[:, ::31] *= 8.0
    return h.cuda(), g


SIZES = [(1, 64), (3, 320), (5, 1024), (2, 1088), (7, 4096), (2, 4160), (3, 16384), (700, 192)]


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16], ids=["f16", "bf16"])
@pytest.mark.parametrize("T,d", SIZES)
@pytest.mark.parametrize("affine", [True, False], ids=["affine", "plain"])
def test_forward(T, d, dtype, affine):
    import paper_2411_01433_amd as P
    h, g = _rows(T, d, T * 31 + d)
    gain = (1 + 0.3 * torch.randn(d, generator=g)).cuda() if affine else None
    bias = (0.3 * torch.randn(d, generator=g)).cuda() if affine else None
    x = torch.full((T + 1, d), 7.0, dtype=dtype, device="cuda")
    P.layernorm(h, x[:T], gain, bias, EPS)
    torch.cuda.synchronize()
    ref = R.layernorm(_f64(h), None if gain is None else _f64(gain),
                      None if bias is None else _f64(bias), EPS)
    n = R.layernorm(_f64(h), eps=EPS)
    H = np.abs(_f64(h)).max(-1, keepdims=True) / np.sqrt(_f64(h).var(-1, keepdims=True) + EPS)
    ga = 1.0 if gain is None else np.abs(_f64(gain))
    tol = HALF[dtype] * np.abs(ref) + 64 * U * (ga * (np.abs(n) + H) + np.abs(ref)) + 2.0 ** -25
    assert (np.abs(_f64(x[:T]) - ref) <= tol).all()
    assert (x[T] == 7.0).all()  # the row behind the last is left as it was


def test_forward_edges():
    """Constant rows (variance 0), a large offset, rows with infinities and NaN,
    whose neighbours stay right, and unaligned lengths of the batch."""
    import paper_2411_01433_amd as P
    d = 256
    h, _ = _rows(6, d, 5)
    h[0] = 3.0
    h[1] = 1000.0 + h[1]
    h[2, 7] = float("inf")
    h[3, 9] = float("nan")
    h[4] = 0.0
    x = torch.empty((6, d), dtype=torch.float16, device="cuda")
    P.layernorm(h, x)
    got = _f64(x)
    assert (got[0] == 0).all() and (got[4] == 0).all()
    assert np.isnan(got[2]).any() and np.isnan(got[3]).all()
    ref = R.layernorm(_f64(h[5:]))
    H = np.abs(_f64(h[5])).max() / _f64(h[5]).std()
    assert (np.abs(got[5:] - ref) <= 2.0 ** -11 * np.abs(ref) + 64 * U * (2 * np.abs(ref) + H) + 2.0 ** -25).all()
    ref = R.layernorm(_f64(h[1:2]))
    H = np.abs(_f64(h[1])).max() / _f64(h[1]).std()
    assert (np.abs(got[1:2] - ref) <= 2.0 ** -11 * np.abs(ref) + 64 * U * (2 * np.abs(ref) + H) + 2.0 ** -25).all()


def _backward_bounds(dx, h, gain, n_adds):
    """(d_h, d_gain, d_bias) bounds for fp32 sums of the given number of steps."""
    dx, h = _f64(dx), _f64(h)
    r = 1.0 / np.sqrt(h.var(-1, keepdims=True) + EPS)
    n = np.abs((h - h.mean(-1, keepdims=True)) * r)
    H = np.abs(h).max(-1, keepdims=True) * r
    a = np.abs(dx) * (1.0 if gain is None else np.abs(_f64(gain)))
    m = lambda v: v.mean(-1, keepdims=True)
    dh = 64 * U * r * (a + m(a) + (n + H) * m(a * (n + H)))
    return dh, n_adds * U * (np.abs(dx) * (n + H)).sum(0), n_adds * U * np.abs(dx).sum(0)


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16], ids=["f16", "bf16"])
@pytest.mark.parametrize("T,d", SIZES + [(2500, 1024), (3000, 64)])
@pytest.mark.parametrize("affine", [True, False], ids=["affine", "plain"])
def test_backward(T, d, dtype, affine):
    import paper_2411_01433_amd as P
    h, g = _rows(T, d, T * 17 + d)
    gain = (1 + 0.3 * torch.randn(d, generator=g)).cuda() if affine else None
    dx = torch.randn((T, d), generator=g).to(dtype).cuda()
    dh = torch.full((T + 1, d), 7.0, device="cuda")
    dg, db = torch.empty(d, device="cuda"), torch.empty(d, device="cuda")
    P.layernorm_backward(dx, h, dh[:T], gain, dg, db, EPS)
    ref = R.layernorm_backward(_f64(dx), _f64(h), None if gain is None else _f64(gain), EPS)
    # a column's sum: at most T / 256 rows of a block, and some tens of joins
    tol = _backward_bounds(dx, h, gain, 96 + T / 256)
    for name, got, want, t in zip(("d_h", "d_gain", "d_bias"), (dh[:T], dg, db), ref, tol):
        off = np.abs(_f64(got) - want)
        assert (off <= t + 2.0 ** -24 * np.abs(want)).all(), (name, (off / t).max())
    assert (dh[T] == 7.0).all()
    # the same bits again; with accumulate the old gradient plus the new one
    again, dg2, db2 = torch.full_like(dh[:T], 2.0), torch.empty_like(dg), torch.empty_like(db)
    P.layernorm_backward(dx, h, again, gain, dg2, db2, EPS, accumulate=True)
    assert torch.equal(again, dh[:T] + 2.0) and torch.equal(dg, dg2) and torch.equal(db, db2)
    # parts of the outputs
    only = torch.empty_like(dg)
    P.layernorm_backward(dx, h, again, gain, None, only, EPS)
    assert torch.equal(only, db) and torch.equal(again, dh[:T])
    P.layernorm_backward(dx, h, again, gain, only, None, EPS)
    assert torch.equal(only, dg)
    P.layernorm_backward(dx, h, again, gain, None, None, EPS)
    assert torch.equal(again, dh[:T])


def test_refusals():
    import paper_2411_01433_amd as P
    h = torch.zeros((4, 128), device="cuda")
    x = torch.zeros((4, 128), dtype=torch.float16, device="cuda")
    v = torch.zeros(128, device="cuda")
    with pytest.raises(ValueError):
        P.layernorm(h, x[:3])
    with pytest.raises(ValueError):
        P.layernorm(h, torch.zeros((4, 128), device="cuda"))
    with pytest.raises(ValueError):
        P.layernorm(h.half(), x)
    with pytest.raises(ValueError):
        P.layernorm(h.t(), x.t())
    with pytest.raises(P.MoeError):
        P.layernorm(h[:, :96].contiguous(), x[:, :96].contiguous())
    with pytest.raises(P.MoeError):
        P.layernorm(h[:0], x[:0])
    with pytest.raises(ValueError, match="bytes"):
        P.layernorm_backward(x, h, h, None, v, v, workspace=torch.empty(16, dtype=torch.uint8, device="cuda"))
    with pytest.raises(ValueError):
        P.layernorm_backward(x, h, h, v[:64], v, v)
    with pytest.raises(P.MoeError, match="aligned"):
        flat = torch.zeros(4 * 128 + 1, device="cuda")
        P.layernorm(flat[1:].view(4, 128), x)


def test_other_stream_and_graph():
    """A call on a side stream, and a captured pass replayed between eager ones
    on new inputs, give the eager bits."""
    import paper_2411_01433_amd as P
    T, d = 300, 512
    h, g = _rows(T, d, 3)
    dx = torch.randn((T, d), generator=g).half().cuda()
    ws = torch.empty(P.layernorm_workspace(T, d), dtype=torch.uint8, device="cuda")
    x = torch.empty((T, d), dtype=torch.float16, device="cuda")
    dh, dg, db = torch.empty_like(h), torch.empty(d, device="cuda"), torch.empty(d, device="cuda")

    def step(stream=None):
        P.layernorm(h, x, None, None, EPS, stream)
        P.layernorm_backward(dx, h, dh, None, dg, db, EPS, workspace=ws, stream=stream)

    def snap():
        torch.cuda.synchronize()
        return [t.clone() for t in (x, dh, dg, db)]

    step()
    ref = snap()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    for t in (x, dh, dg, db):
        t.zero_()
    side.wait_stream(torch.cuda.current_stream())
    step(side)
    assert all(torch.equal(a, b) for a, b in zip(snap(), ref))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    keep = h.clone()
    for i in range(3):
        h.copy_(keep * (i + 2))
        step()
        want = snap()
        for t in (x, dh, dg, db):
            t.zero_()
        graph.replay()
        assert all(torch.equal(a, b) for a, b in zip(snap(), want)), i


def test_offsets_past_32_bits():
    """4.9 GB of rows: the last of them as in a call of their own."""
    import paper_2411_01433_amd as P
    T, d, n = 75000, 16384, 3
    g = torch.Generator(device="cuda").manual_seed(8)
    h = torch.randn((T, d), generator=g, device="cuda")
    gain = torch.randn(d, generator=g, device="cuda")
    x = torch.empty((T, d), dtype=torch.float16, device="cuda")
    P.layernorm(h, x, gain, gain)
    tail = h[-n:].clone()
    own = torch.empty((n, d), dtype=torch.float16, device="cuda")
    P.layernorm(tail, own, gain, gain)
    assert torch.equal(x[-n:], own)
    # gradients of the first and the last rows only: the others add zeros
    dx = x.zero_()
    dx[0] = dx[-n:] = torch.randn(d, generator=g, device="cuda").half()
    dg, db = torch.empty(d, device="cuda"), torch.empty(d, device="cuda")
    dh = torch.empty_like(h)
    P.layernorm_backward(dx, h, dh, gain, dg, db)
    rows = torch.cat([h[:1], tail])
    few, dfew = torch.cat([dx[:1], dx[-n:]]), torch.empty((n + 1, d), device="cuda")
    dg2, db2 = torch.empty(d, device="cuda"), torch.empty(d, device="cuda")
    P.layernorm_backward(few, rows, dfew, gain, dg2, db2)
    assert torch.equal(dh[-n:], dfew[1:]) and torch.equal(dh[:1], dfew[:1])
    # four terms each, in two orders: each order rounds three times to half a step
    norm = (rows - rows.mean(1, keepdim=True)) / rows.std(1, keepdim=True)
    for a, b, terms in ((dg, dg2, few.float() * norm), (db, db2, few.float())):
        assert ((a - b).abs() <= 6 * U * 1.01 * terms.abs().sum(0)).all()
