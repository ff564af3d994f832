"""Grouped products of calls that take the largest blocks: every remainder of
rows and columns, tiles of one stage and of many, blocks that take several
tiles; against float64 on the GPU, with the bounds of the smaller ones: n terms,
S their magnitudes, u = 2^-24 half a step of fp32, n 2 u S element by element, 4
u sqrt(n) of the norm, and half a step of the output's type."""
import numpy as np
import pytest

from oracle import experts_oracle as X

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

U = 2.0 ** -24
HALF = {torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8, torch.float32: U}
TYPES = pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16], ids=["f16", "bf16"])

# every number of 64s in the last tile of an expert, full tiles, none
COUNTS = [1000, 0, 37, 256, 193, 192, 129, 65, 64, 1, 500, 300, 777, 31, 90, 255]
FULL = [1000, 129, 0, 700, 257, 640, 65, 511]


@pytest.fixture(scope="module", autouse=True)
def _need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2411_01433_amd as P
    P.lib()
    yield


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _normal(g, shape, dtype, std=1.0):
    return (std * torch.randn(shape, generator=g, device="cuda")).to(dtype)


def _check(got, ref, S, n, dtype):
    err = (got.double() - ref).abs()
    assert bool((err <= HALF[dtype] * ref.abs() + n * 2 * U * S + 2.0 ** -25).all())
    small = 2.0 ** -25 * ref.numel() ** 0.5 if dtype is torch.float16 else 0.0
    assert float(err.norm()) <= (HALF[dtype] + 4 * U * max(n, 1) ** 0.5) * float(ref.norm()) + small


def _rows(counts, n):
    return [(e, slice(a, a + k)) for e, (a, k) in enumerate(X.expert_rows(counts, n)) if k]


@TYPES
@pytest.mark.parametrize("d_in,d_out", [(64, 6464), (320, 6464), (1088, 6400), (448, 6592), (128, 6336)])
def test_forward(d_in, d_out, dtype):
    import paper_2411_01433_amd as P
    g, R = _gen(d_in), sum(COUNTS)
    x, w = _normal(g, (R + 3, d_in), dtype), _normal(g, (16, d_out, d_in), dtype, 0.05)
    x[R:], w[1] = float("nan"), float("nan")
    y = torch.full((R + 3, d_out), 7.0, dtype=dtype, device="cuda")
    P.grouped_product(x, w, y, torch.tensor(COUNTS, dtype=torch.int32).cuda())
    for e, r in _rows(COUNTS, R):
        a, b = x[r].double(), w[e].double().T
        _check(y[r], a @ b, a.abs() @ b.abs(), d_in, dtype)
    assert bool((y[R:] == 7.0).all())


@TYPES
@pytest.mark.parametrize("d_out,d_in", [(64, 6464), (320, 6464), (1088, 6400), (448, 6592), (128, 6336)])
def test_gradient_of_x(d_in, d_out, dtype):
    import paper_2411_01433_amd as P
    g, R = _gen(d_out), sum(COUNTS)
    dy, w = _normal(g, (R + 3, d_out), dtype, 0.1), _normal(g, (16, d_out, d_in), dtype, 0.05)
    dy[R:], w[1] = float("nan"), float("nan")
    dx = torch.full((R + 3, d_in), 7.0, dtype=dtype, device="cuda")
    P.grouped_product_backward(dy, None, w, torch.tensor(COUNTS, dtype=torch.int32).cuda(), d_x=dx)
    for e, r in _rows(COUNTS, R):
        a, b = dy[r].double(), w[e].double()
        _check(dx[r], a @ b, a.abs() @ b.abs(), d_out, dtype)
    assert bool((dx[R:] == 7.0).all())


@TYPES
@pytest.mark.parametrize("d_in,d_out", [(1600, 2112), (1728, 1984), (2048, 1856)])
def test_gradient_of_w(d_in, d_out, dtype):
    import paper_2411_01433_amd as P
    counts = [0, 1, 63, 64, 65, 700, 0, 128]
    g, R = _gen(d_in), sum(counts)
    x, dy = _normal(g, (R + 2, d_in), dtype), _normal(g, (R + 2, d_out), dtype, 0.1)
    x[R:], dy[R:] = float("nan"), float("nan")
    count = torch.tensor(counts, dtype=torch.int32).cuda()
    dw = torch.full((9, d_out, d_in), 7.0, device="cuda")
    P.grouped_product_backward(dy, x, None, count, d_w=dw[:8])
    base = _normal(g, (8, d_out, d_in), torch.float32)
    more = base.clone()
    P.grouped_product_backward(dy, x, None, count, d_w=more, accumulate=True)
    assert bool(((more - (base + dw[:8])).abs() <= 2 * U * (base + dw[:8]).abs() + 1e-30).all())
    for e, r in _rows(counts, R):
        a, b = dy[r].double().T, x[r].double()
        _check(dw[e], a @ b, a.abs() @ b.abs(), counts[e], torch.float32)
    assert not dw[0].any() and not dw[6].any() and bool((dw[8] == 7.0).all())


def _mx(g, shape, mid=120):
    codes = torch.randint(0, 256, (*shape[:-1], shape[-1] // 2), generator=g, device="cuda", dtype=torch.uint8)
    scales = torch.randint(mid - 6, mid + 7, (*shape[:-1], shape[-1] // 32), generator=g, device="cuda",
                           dtype=torch.uint8)
    return codes, scales


def _values(codes, scales):
    k = torch.stack((codes & 15, codes >> 4), -1).flatten(-2).long()
    v = torch.tensor(X.MX_GRID, device="cuda")[k & 7] * (1.0 - 2.0 * (k >= 8))
    return v * torch.exp2(scales.double() - 127).repeat_interleave(32, -1)


@TYPES
@pytest.mark.parametrize("act", ["16", "4"])
@pytest.mark.parametrize("d_in", [64, 128, 192, 256, 320, 576, 1088])
def test_mx_product(d_in, act, dtype):
    import paper_2411_01433_amd as P
    d_out = 6464
    g, R = _gen(d_in), sum(FULL)
    wc, ws = _mx(g, (8, d_out, d_in))
    ws[2] = 255
    if act == "4":
        x, xs = _mx(g, (R, d_in), 122)
        x64 = _values(x, xs)
    else:
        x, xs = _normal(g, (R, d_in), dtype), None
        x64 = x.double()
    y = torch.full((R + 1, d_out), 7.0, dtype=dtype, device="cuda")
    P.mx_product(x, wc, ws, y[:R], torch.tensor(FULL, dtype=torch.int32).cuda(), xs)
    for e, r in _rows(FULL, R):
        w = _values(wc[e], ws[e]).T
        _check(y[r], x64[r] @ w, x64[r].abs() @ w.abs(), d_in, dtype)
    assert bool((y[R] == 7.0).all())


@pytest.mark.parametrize("counts", [[-5, 3000, -2147483648, 2147483647, 9], [2147483647] * 5, [1, 2, 3, 0, 70],
                                    [4000, 300, 0, 0, 0], [0, 0, 0, 0, 2000]])
def test_counts_that_do_not_fit(counts):
    import paper_2411_01433_amd as P
    R, d_in, d_out = 4097, 128, 6464
    g = _gen(9)
    x, w = _normal(g, (R, d_in), torch.float16), _normal(g, (5, d_out, d_in), torch.float16, 0.05)
    y = torch.full((R + 1, d_out), 7.0, dtype=torch.float16, device="cuda")
    P.grouped_product(x, w, y[:R], torch.tensor(counts, dtype=torch.int32).cuda())
    left = torch.ones(R + 1, dtype=torch.bool, device="cuda")
    for e, r in _rows(counts, R):
        a, b = x[r].double(), w[e].double().T
        _check(y[r], a @ b, a.abs() @ b.abs(), d_in, torch.float16)
        left[r] = False
    assert bool((y[left] == 7.0).all())


def test_two_streams_at_once():
    """Calls share nothing: two that overlap give what each gives alone."""
    import paper_2411_01433_amd as P
    g, R = _gen(3), sum(COUNTS)
    count = torch.tensor(COUNTS, dtype=torch.int32).cuda()
    x, w = _normal(g, (R, 320), torch.float16), _normal(g, (16, 6464, 320), torch.float16, 0.05)
    y = [torch.empty((R, 6464), dtype=torch.float16, device="cuda") for _ in range(3)]
    P.grouped_product(x, w, y[2], count)
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    for _ in range(3):
        for s, out in zip(streams, y):
            P.grouped_product(x, w, out, count, stream=s)
    torch.cuda.synchronize()
    assert torch.equal(y[0], y[2]) and torch.equal(y[1], y[2])
