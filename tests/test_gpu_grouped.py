"""Products grouped by expert and their backward pass against the float64
oracle.

Bounds.  u = 2^-24 is half a step of fp32, S the sum of the magnitudes of an
output's n terms.  Products of two 16-bit numbers are exact in fp32; every
addition is off by at most a step (2 u) of a partial sum, which is at most S:
n 2 u S in all, whatever the order.  That is far more than rounding that is as
often up as down leaves, so the whole output is held to 4 u sqrt(n) of its norm
besides.  The rounding to the output's type adds half a step of it (and half
of the smallest subnormal of fp16)."""
import numpy as np
import pytest

from oracle import experts_oracle as X

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

U = 2.0 ** -24
HALF = {torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8, torch.float32: U}
TYPES = pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16], ids=["f16", "bf16"])


@pytest.fixture(scope="module", autouse=True)
def _need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2411_01433_amd as P
    P.lib()
    yield


def _f64(t):
    return t.double().cpu().numpy()


def _normal(g, shape, dtype, std=1.0):
    return (std * torch.randn(shape, generator=g)).to(dtype).cuda()


def _check(got, ref, S, n, dtype):
    """n: terms of each output, a number or per row."""
    err = np.abs(got - ref)
    n = np.broadcast_to(np.asarray(n, np.float64).reshape(-1, *[1] * (ref.ndim - 1)), ref.shape)
    assert (err <= HALF[dtype] * np.abs(ref) + n * 2 * U * S + 2.0 ** -25).all()
    norm = np.linalg.norm(ref)
    # (subnormals of fp16 are rounded by more than their relative half step)
    small = 2.0 ** -25 * np.sqrt(ref.size) if dtype is torch.float16 else 0.0
    assert np.linalg.norm(err) <= (HALF[dtype] + 4 * U * np.sqrt(n.max(initial=1))) * norm + small


# counts of the experts, d_in, d_out, rows behind the last expert's
CASES = [
    ([1], 64, 64, 0),
    ([0, 3, 0, 1], 64, 128, 2),
    ([2, 0, 0, 0, 0, 0, 0, 0], 1024, 2048, 0),
    ([0, 1, 0, 0, 0, 1, 0, 0], 2048, 704, 1),
    ([5, 0, 17, 33, 64, 65], 320, 448, 3),
    ([15, 16, 17, 31, 32, 1], 448, 192, 0),
    ([200, 1, 0, 255, 256, 257], 192, 320, 5),
    ([513, 127, 129], 128, 576, 0),
    ([1300], 128, 704, 0),
    ([700, 0, 41], 1088, 64, 1),
    ([0] * 8, 128, 64, 4),
    ([(7 * e * e + 3 * e) % 23 for e in range(60)], 256, 320, 0),
    ([e % 3 for e in range(512)], 64, 64, 7),
    ([0] * 511 + [70], 64, 192, 0),
]
IDS = [f"e{len(c[0])}_r{sum(c[0])}_{c[1]}x{c[2]}" for c in CASES]
SIZES = pytest.mark.parametrize("counts,d_in,d_out,extra", CASES, ids=IDS)


def _inputs(counts, d_in, d_out, extra, dtype):
    R, E = sum(counts) + extra, len(counts)
    g = torch.Generator().manual_seed(R * 31 + d_in + d_out)
    x = _normal(g, (R, d_in), dtype)
    w = _normal(g, (E, d_out, d_in), dtype, 0.05)
    dy = _normal(g, (R, d_out), dtype, 0.1)
    # neither the rows behind the last nor an unused expert may be read
    for t in (x, dy):
        t[sum(counts):] = float("nan")
    for e, c in enumerate(counts):
        if c == 0:
            w[e] = float("nan")
    return x, w, dy, torch.tensor(counts, dtype=torch.int32).cuda()


def _clean(t):
    return np.nan_to_num(_f64(t))


@TYPES
@SIZES
def test_forward(counts, d_in, d_out, extra, dtype):
    import paper_2411_01433_amd as P
    x, w, _, count = _inputs(counts, d_in, d_out, extra, dtype)
    y = torch.full((x.shape[0], d_out), 7.0, dtype=dtype, device="cuda")
    P.grouped_product(x, w, y, count)
    ref, S = X.grouped_product(_clean(x), _clean(w), counts, np.full(tuple(y.shape), 7.0))
    n = sum(counts)
    assert (y[n:] == 7.0).all()
    _check(_f64(y)[:n], ref[:n], S[:n], d_in, dtype)
    again = torch.empty_like(y)
    P.grouped_product(x, w, again, count)
    assert torch.equal(again[:n], y[:n])
    if len(counts) == 1:
        again.zero_()
        P.grouped_product(x[:n], w, again[:n])
        assert torch.equal(again[:n], y[:n])


@TYPES
@SIZES
def test_backward(counts, d_in, d_out, extra, dtype):
    import paper_2411_01433_amd as P
    x, w, dy, count = _inputs(counts, d_in, d_out, extra, dtype)
    dx = torch.full_like(x, 7.0)
    dw = torch.full(w.shape, 7.0, device="cuda")
    P.grouped_product_backward(dy, x, w, count, dx, dw)
    rx, rw, sx, sw = X.grouped_product_backward(_clean(dy), _clean(x), _clean(w), counts,
                                                np.full(tuple(x.shape), 7.0), np.zeros(tuple(w.shape)))
    n = sum(counts)
    assert (dx[n:] == 7.0).all()
    _check(_f64(dx)[:n], rx[:n], sx[:n], d_out, dtype)
    _check(_f64(dw), rw, sw, counts, torch.float32)
    # each alone, and added to what is there
    dx1, dw1 = torch.full_like(x, 7.0), torch.empty_like(dw)
    P.grouped_product_backward(dy, None, w, count, d_x=dx1)
    P.grouped_product_backward(dy, x, None, count, d_w=dw1)
    assert torch.equal(dx1, dx) and torch.equal(dw1, dw)
    g = torch.Generator().manual_seed(1)
    base = _normal(g, w.shape, torch.float32)
    dw1.copy_(base)
    P.grouped_product_backward(dy, x, None, count, d_w=dw1, accumulate=True)
    assert ((dw1 - (base + dw)).abs() <= 2 * U * (base + dw).abs() + 1e-30).all()


WIDE = pytest.mark.parametrize("counts,extra", [
    ([70, 0, 128, 129, 33, 255, 1, 64], 3),
    ([(11 * e) % 40 for e in range(20)], 0),
    ([260], 1),
])


@TYPES
@WIDE
@pytest.mark.parametrize("d_in,d_out", [(192, 2112), (2112, 192), (5568, 5504)])
def test_wide_rows(counts, extra, d_in, d_out, dtype):
    """More tiles than the calls above have, of columns of y and of d_x."""
    if d_in * d_out * len(counts) > 8 * 5568 * 2112:
        counts, extra = [90], 0
    test_forward(counts, d_in, d_out, extra, dtype)
    test_backward(counts, d_in, d_out, extra, dtype)


@pytest.mark.parametrize("counts", [[-3, 5, -2147483648, 2], [4, 2147483647, 3],
                                    [2147483647] * 4, [20, 0, 0, 0], [3, 9, 1, 1]])
def test_counts_that_do_not_fit(counts):
    """A negative count is no row; what lies behind n_rows is cut."""
    import paper_2411_01433_amd as P
    R, d_in, d_out, E = 11, 128, 192, len(counts)
    g = torch.Generator().manual_seed(3)
    x, dy = _normal(g, (R, d_in), torch.float16), _normal(g, (R, d_out), torch.float16, 0.1)
    w = _normal(g, (E, d_out, d_in), torch.float16, 0.05)
    count = torch.tensor(counts, dtype=torch.int32).cuda()
    y = torch.full((R + 1, d_out), 7.0, dtype=torch.float16, device="cuda")
    dx = torch.full((R + 1, d_in), 7.0, dtype=torch.float16, device="cuda")
    dw = torch.full((E + 1, d_out, d_in), 7.0, device="cuda")
    P.grouped_product(x, w, y[:R], count)
    P.grouped_product_backward(dy, x, w, count, dx[:R], dw[:E])
    ref, S = X.grouped_product(_f64(x), _f64(w), counts, np.full((R, d_out), 7.0))
    rx, rw, sx, sw = X.grouped_product_backward(_f64(dy), _f64(x), _f64(w), counts,
                                                np.full((R, d_in), 7.0), np.zeros((E, d_out, d_in)))
    _check(_f64(y)[:R], ref, S, d_in, torch.float16)
    _check(_f64(dx)[:R], rx, sx, d_out, torch.float16)
    _check(_f64(dw)[:E], rw, sw, R, torch.float32)
    assert (y[R] == 7.0).all() and (dx[R] == 7.0).all() and (dw[E] == 7.0).all()


def test_no_rows():
    import paper_2411_01433_amd as P
    x = torch.empty((0, 64), dtype=torch.bfloat16, device="cuda")
    w = torch.full((3, 128, 64), float("nan"), dtype=torch.bfloat16, device="cuda")
    y = torch.empty((0, 128), dtype=torch.bfloat16, device="cuda")
    count = torch.zeros(3, dtype=torch.int32, device="cuda")
    dw = torch.full((3, 128, 64), 7.0, device="cuda")
    P.grouped_product(x, w, y, count)
    P.grouped_product_backward(y, x, w, count, x, dw, accumulate=True)
    assert (dw == 7.0).all()
    P.grouped_product_backward(y, x, w, count, x, dw)
    assert (dw == 0.0).all()


@TYPES
def test_infinities_stay_in_their_rows(dtype):
    """An infinity or NaN in a row of x enters that row of y only, and of the
    weights' gradient that of its expert; zeros beside it stay exact."""
    import paper_2411_01433_amd as P
    counts, d_in, d_out = [70, 3, 150], 192, 128
    x, w, dy, count = _inputs(counts, d_in, d_out, 0, dtype)
    y0, y1 = (torch.empty((223, d_out), dtype=dtype, device="cuda") for _ in range(2))
    dx0, dx1 = torch.empty_like(x), torch.empty_like(x)
    dw0, dw1 = (torch.empty((3, d_out, d_in), device="cuda") for _ in range(2))
    P.grouped_product(x, w, y0, count)
    P.grouped_product_backward(dy, x, w, count, dx0, dw0)
    x[71, 5], x[60, 191], dy[100, 7] = float("inf"), float("nan"), float("-inf")
    P.grouped_product(x, w, y1, count)
    P.grouped_product_backward(dy, x, w, count, dx1, dw1)
    hit = torch.zeros(223, dtype=torch.bool, device="cuda")
    hit[[60, 71]] = True
    assert torch.equal(y1[~hit], y0[~hit]) and not torch.isfinite(y1[hit]).any()
    hit.zero_()
    hit[100] = True
    assert torch.equal(dx1[~hit], dx0[~hit]) and not torch.isfinite(dx1[hit]).any()
    # column 191 of expert 0, column 5 of expert 1, row 7 of expert 2
    bad = torch.zeros(dw1.shape, dtype=torch.bool, device="cuda")
    bad[0, :, 191] = bad[1, :, 5] = bad[2, 7] = True
    assert torch.equal(dw1[~bad], dw0[~bad]) and not torch.isfinite(dw1[bad]).any()


def test_rounding_to_the_type():
    """Sums beyond fp16 go to infinity, subnormal ones are kept."""
    import paper_2411_01433_amd as P
    x = torch.full((1, 64), 128.0, dtype=torch.float16, device="cuda")
    w = torch.zeros((1, 64, 64), dtype=torch.float16, device="cuda")
    w[0, 0], w[0, 1], w[0, 2, 0], w[0, 3, 0] = 128.0, 7.9921875, 2.0 ** -24, -(2.0 ** -24)
    y = torch.empty((1, 64), dtype=torch.float16, device="cuda")
    P.grouped_product(x, w, y)
    assert y[0, 0] == float("inf") and y[0, 1] == 65472.0
    assert y[0, 2] == 2.0 ** -17 and y[0, 3] == -(2.0 ** -17) and (y[0, 4:] == 0).all()
    x.fill_(2.0 ** -24)
    w[0, 0] = 1.0
    P.grouped_product(x, w, y)
    assert y[0, 0] == 2.0 ** -18


def test_gradients_against_differences():
    """The derivative of sum(dy * y) along random directions of x and of W, from
    y of both sides: y is linear in either, so the difference is exact up to
    the rounding of y (fp16 inputs on a coarse grid: products and sums exact)."""
    import paper_2411_01433_amd as P
    g = torch.Generator().manual_seed(5)
    counts, d_in, d_out = [9, 0, 40], 64, 128
    R = sum(counts)
    grid = lambda *s: (torch.randint(-4, 5, s, generator=g).double() / 4).half().cuda()
    x, w, dy = grid(R, d_in), grid(3, d_out, d_in), grid(R, d_out)
    vx, vw = grid(R, d_in), grid(3, d_out, d_in)
    count = torch.tensor(counts, dtype=torch.int32).cuda()
    dx, dw = torch.empty_like(x), torch.empty(w.shape, device="cuda")
    P.grouped_product_backward(dy, x, w, count, dx, dw)

    def loss(x, w):
        y = torch.empty((R, d_out), dtype=torch.float16, device="cuda")
        P.grouped_product(x, w, y, count)
        return (dy.double() * y.double()).sum()

    # values are multiples of 1/16 below 64 * 2 = 128: 11 bits hold them all
    for at, da, v, f in ((x, dx, vx, lambda t: loss(t, w)), (w, dw, vw, lambda t: loss(x, t))):
        diff = f(at + v) - f(at - v)
        used = v.double()
        if at is w:
            used[1] = 0.0
        assert abs(diff / 2 - (da.double() * used).sum()) <= 1e-9 * (dy.double().abs().sum() * 128)


def test_binding_refuses():
    import paper_2411_01433_amd as P
    x = torch.zeros((4, 64), dtype=torch.float16, device="cuda")
    w = torch.zeros((2, 128, 64), dtype=torch.float16, device="cuda")
    y = torch.zeros((4, 128), dtype=torch.float16, device="cuda")
    dw = torch.zeros((2, 128, 64), device="cuda")
    n = torch.zeros(2, dtype=torch.int32, device="cuda")
    for bad in (lambda: P.grouped_product(x.float(), w, y, n), lambda: P.grouped_product(x, w.bfloat16(), y, n),
                lambda: P.grouped_product(x, w, y.bfloat16(), n), lambda: P.grouped_product(x, w, y[:3], n),
                lambda: P.grouped_product(x, w, y, n.long()), lambda: P.grouped_product(x, w, y, n[:1]),
                lambda: P.grouped_product(x.cpu(), w, y, n), lambda: P.grouped_product(x, w[0], y, n),
                lambda: P.grouped_product(x[:, ::2], w, y, n),
                lambda: P.grouped_product(x, w.transpose(1, 2), y, n),
                lambda: P.grouped_product_backward(y, x, w, n),
                lambda: P.grouped_product_backward(y, None, w, n, d_w=dw),
                lambda: P.grouped_product_backward(y, x, None, n, d_x=x),
                lambda: P.grouped_product_backward(y, x, w, n, d_w=dw.half())):
        with pytest.raises(ValueError):
            bad()
    with pytest.raises(P.MoeError):
        P.grouped_product(x, w, y)  # two experts without counts


def _graph_inputs():
    counts = [33, 0, 5, 90]
    return _inputs(counts, 192, 256, 1, torch.float16)


def test_captured_and_on_another_stream():
    """Forward and backward in a graph, replayed with new counts and inputs, with
    eager calls on another stream between the replays."""
    import paper_2411_01433_amd as P
    x, w, dy, count = _graph_inputs()
    w.nan_to_num_(0.1)
    y = torch.zeros((x.shape[0], 256), dtype=torch.float16, device="cuda")
    dx, dw = torch.zeros_like(x), torch.zeros(w.shape, device="cuda")
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        P.grouped_product(x, w, y, count)
        P.grouped_product_backward(dy, x, w, count, dx, dw)
    side = torch.cuda.Stream()
    for counts in ([33, 0, 5, 90], [0, 0, 0, 0], [128, 0, 0, 0], [1, 60, 60, 7]):
        count.copy_(torch.tensor(counts, dtype=torch.int32))
        x[:128].mul_(0.9)
        y.zero_(), dx.zero_()
        y2, dx2, dw2 = torch.zeros_like(y), torch.zeros_like(dx), torch.empty_like(dw)
        graph.replay()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            P.grouped_product(x, w, y2, count)
            P.grouped_product_backward(dy, x, w, count, dx2, dw2)
        torch.cuda.synchronize()
        P.grouped_product(x, w, torch.empty_like(y), count)
        assert torch.equal(y, y2) and torch.equal(dx, dx2) and torch.equal(dw, dw2)


def test_rows_past_4_gib():
    """x and W of more than 2^32 elements: the last rows and the last expert."""
    import paper_2411_01433_amd as P
    g = torch.Generator().manual_seed(8)
    E, R, d_in, d_out = 512, 1 << 21, 2112, 64
    x = torch.zeros((R, d_in), dtype=torch.float16, device="cuda")
    x[-40:] = _normal(g, (40, d_in), torch.float16)
    w = torch.zeros((E, d_out, d_in), dtype=torch.float16, device="cuda")
    w[-1] = _normal(g, (d_out, d_in), torch.float16, 0.05)
    counts = [0] * E
    counts[1], counts[-1] = R - 37, 37
    count = torch.tensor(counts, dtype=torch.int32).cuda()
    y = torch.empty((R, d_out), dtype=torch.float16, device="cuda")
    P.grouped_product(x, w, y, count)
    ref, S = X.grouped_product(_f64(x[-37:]), _f64(w[-1:]), [37], np.zeros((37, d_out)))
    _check(_f64(y[-37:]), ref, S, d_in, torch.float16)
    assert not y[:-37].any()
    dy = torch.zeros((R, d_out), dtype=torch.float16, device="cuda")
    dy[-37:] = _normal(g, (37, d_out), torch.float16, 0.1)
    dw = torch.empty((E, d_out, d_in), device="cuda")
    x1 = x[-37:].clone()
    P.grouped_product_backward(dy, x, w, count, d_w=dw)
    P.grouped_product_backward(dy, None, w, count, d_x=x)
    rx, rw, sx, sw = X.grouped_product_backward(_f64(dy[-37:]), _f64(x1), _f64(w[-1:]), [37],
                                                np.zeros((37, d_in)), np.zeros((1, d_out, d_in)))
    _check(_f64(x[-37:]), rx, sx, d_out, torch.float16)
    _check(_f64(dw[-1:]), rw, sw, 37, torch.float32)
    assert not dw[:-1].any()
    del x
    # the weights themselves past 4 GiB
    E, d_in, d_out = 5, 65536, 16384
    w = torch.zeros((E, d_out, d_in), dtype=torch.float16, device="cuda")
    w[-1, -3:] = _normal(g, (3, d_in), torch.float16, 0.05)
    x = _normal(g, (3, d_in), torch.float16)
    count = torch.tensor([0, 0, 0, 0, 3], dtype=torch.int32).cuda()
    y = torch.empty((3, d_out), dtype=torch.float16, device="cuda")
    P.grouped_product(x, w, y, count)
    ref, S = X.grouped_product(_f64(x), _f64(w[-1:, -3:]), [3], np.zeros((3, 3)))
    _check(_f64(y[:, -3:]), ref, S, d_in, torch.float16)
    assert not y[:, :-3].any()
    dy = torch.zeros((3, d_out), dtype=torch.float16, device="cuda")
    dy[:, -3:] = _normal(g, (3, 3), torch.float16)
    dx = torch.empty_like(x)
    dw = torch.empty(w.shape, device="cuda")
    P.grouped_product_backward(dy, x, w, count, dx, dw)
    rx, rw, sx, sw = X.grouped_product_backward(_f64(dy[:, -3:]), _f64(x), _f64(w[-1:, -3:]), [3],
                                                np.zeros((3, d_in)), np.zeros((1, 3, d_in)))
    _check(_f64(dx), rx, sx, d_out, torch.float16)
    _check(_f64(dw[-1:, -3:]), rw, sw, 3, torch.float32)
    assert not dw[:-1].any() and not dw[-1, :-3].any()
