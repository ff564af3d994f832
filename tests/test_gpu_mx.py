"""The MXFP4 quantiser and its products against the float64 oracle.  Codes,
scales and values match exactly; the products' bounds are those of the grouped
products (n terms, S their magnitudes): n 2 u S element by element, 4 u sqrt(n)
of the norm, and half a step of the output's type.  Products of two codes and
their scales are exact, as are those of a code and a 16-bit number."""
import numpy as np
import pytest

from oracle import experts_oracle as X

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

U = 2.0 ** -24
HALF = {torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}
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


def _quantize(v, values=None):
    import paper_2411_01433_amd as P
    rows, cols = v.shape
    codes = torch.full((rows, cols // 2), 0xEE, dtype=torch.uint8, device="cuda")
    scales = torch.full((rows, cols // 32), 0xEE, dtype=torch.uint8, device="cuda")
    P.mx_quantize(v, codes, scales, values)
    return codes, scales


def _check_quantized(v):
    values = torch.empty_like(v)
    codes, scales = _quantize(v, values)
    rc, rs = X.mx_quantize(_f64(v))
    assert (scales.cpu().numpy() == rs).all()
    assert (codes.cpu().numpy() == rc).all()
    assert (_f64(values) == X.mx_values(rc, rs)).all()


@TYPES
@pytest.mark.parametrize("rows,cols", [(1, 64), (3, 320), (1, 4096), (129, 448), (1000, 64),
                                       (2, 65536), (333, 1088)])
def test_quantize(rows, cols, dtype):
    g = torch.Generator().manual_seed(rows + cols)
    v = torch.randn((rows, cols), generator=g) * torch.exp(2 * torch.randn((rows, cols // 32, 1), generator=g)).expand(-1, -1, 32).reshape(rows, cols)
    _check_quantized(v.to(dtype).cuda())


@TYPES
def test_quantize_every_number(dtype):
    """Every finite bit pattern: in blocks of neighbours, and beside each power of
    two that can set the block's scale (so that ties and saturation are met)."""
    bits = np.arange(65536, dtype=np.uint16)
    v = torch.from_numpy(bits.view(np.int16)).view(dtype)
    v = v[torch.isfinite(v)]
    _check_quantized(v.view(-1, 64).cuda())
    lead = torch.exp2(torch.arange(-24, 16) if dtype is torch.float16 else torch.arange(-133, 128)).to(dtype)
    for top in (1.0, 1.5, 1.75, 1.9375):
        rows = []
        for p in lead.double():
            if p * top > torch.finfo(dtype).max:
                continue
            k = torch.arange(62).double() / 62 * 8  # up to the block's top
            q = torch.cat((k, torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 7.0]).double()))
            row = (torch.cat((q, -q))[:124] * p / 4).to(dtype)
            full = torch.zeros(4 * 32, dtype=dtype)
            full.view(4, 32)[:, 1:] = row.view(4, 31)
            full.view(4, 32)[:, 0] = (p * top).to(dtype)
            rows.append(full)
        _check_quantized(torch.stack(rows).cuda())


@TYPES
def test_quantize_not_finite(dtype):
    """A block with an infinity or NaN is NaN; its neighbours are not."""
    g = torch.Generator().manual_seed(1)
    v = torch.randn((4, 128), generator=g).to(dtype)
    rc, rs = X.mx_quantize(v.double().numpy())
    v[0, 40], v[1, 0], v[3, 127] = float("inf"), float("nan"), float("-inf")
    rs[0, 1] = rs[1, 0] = rs[3, 3] = 255
    values = torch.empty_like(v).cuda()
    codes, scales = _quantize(v.cuda(), values)
    assert (scales.cpu().numpy() == rs).all()
    ok = np.repeat(rs != 255, 16, -1)
    assert (codes.cpu().numpy()[ok] == rc[ok]).all()
    ref = X.mx_values(rc, rs)
    assert np.array_equal(_f64(values), ref, equal_nan=True)


def test_quantize_in_place_and_no_rows():
    import paper_2411_01433_amd as P
    g = torch.Generator().manual_seed(2)
    v = torch.randn((70, 192), generator=g).half().cuda()
    want = torch.empty_like(v)
    codes, scales = _quantize(v, want)
    got = v.clone()
    c2, s2 = _quantize(got, got)
    assert torch.equal(got, want) and torch.equal(codes, c2) and torch.equal(scales, s2)
    e = lambda *s: torch.empty(s, dtype=torch.uint8, device="cuda")
    P.mx_quantize(v[:0], e(0, 96), e(0, 6))


def test_quantize_past_4_gib():
    rows, cols = 65537, 65536
    v = torch.zeros((rows, cols), dtype=torch.float16, device="cuda")
    g = torch.Generator().manual_seed(3)
    v[-1] = torch.randn(cols, generator=g).half().cuda()
    codes, scales = _quantize(v, v)
    rc, rs = X.mx_quantize(torch.randn(1, cols, generator=torch.Generator().manual_seed(3)).half().double().numpy())
    assert (codes[-1].cpu().numpy() == rc[0]).all() and (scales[-1].cpu().numpy() == rs[0]).all()
    assert not codes[:-1].any() and not scales[:-1].any()
    assert (_f64(v[-1]) == X.mx_values(rc, rs)[0]).all()


# ---- products -------------------------------------------------------------------

def _check(got, ref, S, n, dtype):
    err = np.abs(got - ref)
    assert (err <= HALF[dtype] * np.abs(ref) + n * 2 * U * S + 2.0 ** -25).all()
    small = 2.0 ** -25 * np.sqrt(ref.size) if dtype is torch.float16 else 0.0
    assert np.linalg.norm(err) <= (HALF[dtype] + 4 * U * np.sqrt(n)) * np.linalg.norm(ref) + small


def _mx_matrix(shape, seed, spread=6, mid=120):
    """Random codes, with scales of some binades."""
    r = np.random.default_rng(seed)
    codes = r.integers(0, 256, (*shape[:-1], shape[-1] // 2), dtype=np.uint8)
    scales = r.integers(mid - spread, mid + spread + 1, (*shape[:-1], shape[-1] // 32)).astype(np.uint8)
    return codes, scales


CASES = [
    ([1], 64, 64, 0),
    ([0, 3, 0, 1], 128, 128, 2),
    ([2, 0, 0, 0, 0, 0, 0, 0], 1024, 2048, 0),
    ([0, 1, 0, 0, 0, 1, 0, 0], 2048, 704, 1),
    ([5, 0, 17, 33, 64, 65], 320, 448, 3),
    ([15, 16, 17, 31, 32, 1], 448, 192, 0),
    ([200, 1, 0, 255, 256, 257], 192, 320, 5),
    ([513, 127, 129], 576, 576, 0),
    ([1300], 64, 704, 0),
    ([700, 0, 41], 1088, 64, 1),
    ([0] * 8, 128, 64, 4),
    ([(7 * e * e + 3 * e) % 23 for e in range(60)], 256, 320, 0),
    ([e % 3 for e in range(512)], 64, 64, 7),
    ([400, 300], 832, 320, 0),
]
IDS = [f"e{len(c[0])}_r{sum(c[0])}_{c[1]}x{c[2]}" for c in CASES]


@pytest.mark.parametrize("act", ["16", "4"])
@TYPES
@pytest.mark.parametrize("counts,d_in,d_out,extra", CASES, ids=IDS)
def test_product(counts, d_in, d_out, extra, dtype, act):
    import paper_2411_01433_amd as P
    R, E, n = sum(counts) + extra, len(counts), sum(counts)
    codes, scales = _mx_matrix((E, d_out, d_in), R + d_in)
    w = X.mx_values(codes, scales)
    for e, c in enumerate(counts):  # an unused expert is not read
        if c == 0:
            scales[e] = 255
    wc, ws = torch.from_numpy(codes).cuda(), torch.from_numpy(scales).cuda()
    count = torch.tensor(counts, dtype=torch.int32).cuda()
    y = torch.full((R, d_out), 7.0, dtype=dtype, device="cuda")
    if act == "4":
        xc, xs = _mx_matrix((R, d_in), R, 8, 122)
        x64 = X.mx_values(xc, xs)
        xs[n:] = 255
        x, x_scales = torch.from_numpy(xc).cuda(), torch.from_numpy(xs).cuda()
    else:
        g = torch.Generator().manual_seed(R)
        x = torch.randn((R, d_in), generator=g).to(dtype).cuda()
        x64, x_scales = _f64(x), None
        x[n:] = float("nan")
    P.mx_product(x, wc, ws, y, count, x_scales)
    ref, S = X.grouped_product(x64, w, counts, np.full((R, d_out), 7.0))
    assert (y[n:] == 7.0).all()
    _check(_f64(y)[:n], ref[:n], S[:n], d_in, dtype)
    again = torch.empty_like(y)
    P.mx_product(x, wc, ws, again, count, x_scales)
    assert torch.equal(again[:n], y[:n])
    if E == 1:
        P.mx_product(x, wc, ws, again, None, x_scales)  # (takes the rows behind too)
        assert torch.equal(again[:n], y[:n])


@pytest.mark.parametrize("act", ["16", "4"])
@pytest.mark.parametrize("counts,d_in,d_out,extra", [
    ([1], 8192, 64, 0),
    ([3, 0, 16, 0, 1], 8256, 192, 2),
    ([0, 2, 11], 20544, 128, 0),
    ([40], 16448, 192, 1),
    ([0] * 7 + [61], 448, 192, 2),
    ([14], 448, 64, 0),
    ([3, 45, 17], 1088, 192, 0),
])
def test_rows_of_many_columns(counts, d_in, d_out, extra, act):
    """Blocks whose waves share the columns, and several slabs of them."""
    test_product(counts, d_in, d_out, extra, torch.bfloat16, act)


@pytest.mark.parametrize("act", ["16", "4"])
@TYPES
@pytest.mark.parametrize("counts,extra", [
    ([70, 0, 128, 129, 33, 255, 1, 64], 3),
    ([(11 * e) % 40 for e in range(20)], 0),
    ([520], 1),
])
@pytest.mark.parametrize("d_in,d_out", [(192, 2112), (832, 3520)])
def test_wide_rows(counts, extra, d_in, d_out, dtype, act):
    """More tiles than the calls above have."""
    test_product(counts, d_in, d_out, extra, dtype, act)


@pytest.mark.parametrize("rows", [1, 3, 40, 300])
def test_scales_over_the_whole_range(rows):
    """Scale bytes 0 (2^-127) to 254 in bf16 and 4-bit products, whose partner
    brings the result back into range; with x in fp16 all that fp16 holds."""
    import paper_2411_01433_amd as P
    d_in, d_out = 256, 64
    r = np.random.default_rng(rows)
    codes = r.integers(0, 256, (1, d_out, d_in // 2), dtype=np.uint8)
    e = np.array([0, 1, 2, 100, 127, 150, 200, 250] * (d_out // 8)).astype(np.uint8)
    scales = np.repeat(e.reshape(1, d_out, 1), d_in // 32, -1)
    w = X.mx_values(codes, scales)
    # one size of x for all: outputs outside of the range are left out below
    for byte in (254, 130, 60):
        xc = r.integers(0, 256, (rows, d_in // 2), dtype=np.uint8)
        xs = np.full((rows, d_in // 32), byte, np.uint8)
        x64 = X.mx_values(xc, xs)
        big = np.abs(x64) * np.ldexp(1.0, -127) > 2.0 ** 0.9  # 6 2^127 is beyond bf16
        y = torch.empty((rows, d_out), dtype=torch.bfloat16, device="cuda")
        P.mx_product(torch.from_numpy(xc).cuda(), torch.from_numpy(codes).cuda(),
                     torch.from_numpy(scales).cuda(), y, None, torch.from_numpy(xs).cuda())
        ref, S = X.grouped_product(x64, w, [rows], np.zeros((rows, d_out)))
        ok = (S < 2.0 ** 126) & (S > 2.0 ** -90)
        got = _f64(y)
        assert ok.any() and (np.abs(got - ref) <= HALF[torch.bfloat16] * np.abs(ref) + d_in * 2 * U * S)[ok].all()
        if not big.any():
            xb = torch.from_numpy(x64).bfloat16().cuda()
            P.mx_product(xb, torch.from_numpy(codes).cuda(), torch.from_numpy(scales).cuda(), y)
            got = _f64(y)
            assert (np.abs(got - ref) <= HALF[torch.bfloat16] * np.abs(ref) + d_in * 2 * U * S)[ok].all()
    # fp16: 2^-23 .. 2^13 (bytes 104 .. 140) are exact, 2^-24 loses the code 0.5's half
    scales = np.repeat(np.array([104, 110, 120, 127, 130, 135, 139, 140] * (d_out // 8)).astype(np.uint8).reshape(1, d_out, 1), d_in // 32, -1)
    w = X.mx_values(codes, scales)
    x = torch.from_numpy(r.standard_normal((rows, d_in)) * 2.0 ** -8).half().cuda()
    y = torch.empty((rows, d_out), dtype=torch.float16, device="cuda")
    P.mx_product(x, torch.from_numpy(codes).cuda(), torch.from_numpy(scales).cuda(), y)
    ref, S = X.grouped_product(_f64(x), w, [rows], np.zeros((rows, d_out)))
    ok = S < 60000
    assert (np.abs(_f64(y) - ref) <= 2.0 ** -11 * np.abs(ref) + d_in * 2 * U * S + 2.0 ** -25)[ok].all()


@pytest.mark.parametrize("act", ["16", "4"])
@pytest.mark.parametrize("rows", [2, 90])
def test_nan_scales_stay_in_their_outputs(rows, act):
    import paper_2411_01433_amd as P
    d_in, d_out = 320, 192
    codes, scales = _mx_matrix((1, d_out, d_in), 4)
    scales[0, 100, 9] = 255
    wc, ws = torch.from_numpy(codes).cuda(), torch.from_numpy(scales).cuda()
    if act == "4":
        xc, xs = _mx_matrix((rows, d_in), 5)
        xs[1, 0] = 255
        x, x_scales = torch.from_numpy(xc).cuda(), torch.from_numpy(xs).cuda()
    else:
        x, x_scales = torch.ones((rows, d_in), dtype=torch.bfloat16, device="cuda"), None
        x[1, 3] = float("nan")
    y = torch.empty((rows, d_out), dtype=torch.bfloat16, device="cuda")
    P.mx_product(x, wc, ws, y, None, x_scales)
    nan = torch.isnan(y)
    want = torch.zeros_like(nan)
    want[:, 100] = True
    want[1] = True
    assert torch.equal(nan, want)


def test_quantized_weights_multiply_as_their_values():
    """The product with quantised weights is the grouped product with the values
    that the quantiser returns, up to the order of sums; and with x quantised
    too that of both values."""
    import paper_2411_01433_amd as P
    g = torch.Generator().manual_seed(6)
    counts, d_in, d_out = [3, 0, 100], 384, 256
    w = (0.02 * torch.randn((3 * d_out, d_in), generator=g)).half().cuda()
    x = torch.randn((103, d_in), generator=g).half().cuda()
    wv, xv = torch.empty_like(w), torch.empty_like(x)
    wc, ws = _quantize(w, wv)
    xc, xs = _quantize(x, xv)
    count = torch.tensor(counts, dtype=torch.int32).cuda()
    y = torch.empty((103, d_out), dtype=torch.float16, device="cuda")
    args = wc.view(3, d_out, -1), ws.view(3, d_out, -1), y, count
    for x1, xq, s in ((x, x, None), (xv, xc, xs)):
        P.mx_product(xq, *args, s)
        ref, S = X.grouped_product(_f64(x1), _f64(wv).reshape(3, d_out, d_in), counts, np.zeros((103, d_out)))
        _check(_f64(y), ref, S, d_in, torch.float16)


def test_captured():
    import paper_2411_01433_amd as P
    g = torch.Generator().manual_seed(7)
    counts, d_in, d_out = [3, 0, 100], 384, 256
    w = (0.02 * torch.randn((3 * d_out, d_in), generator=g)).half().cuda()
    x = torch.randn((103, d_in), generator=g).half().cuda()
    wc, ws = _quantize(w)
    wc, ws = wc.view(3, d_out, -1), ws.view(3, d_out, -1)
    xc, xs = _quantize(x)
    count = torch.tensor(counts, dtype=torch.int32).cuda()
    y4, y16 = (torch.empty((103, d_out), dtype=torch.float16, device="cuda") for _ in range(2))
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        P.mx_quantize(x, xc, xs)
        P.mx_product(xc, wc, ws, y4, count, xs)
        P.mx_product(x, wc, ws, y16, count)
    for _ in range(3):
        x.mul_(1.3)
        graph.replay()
        torch.cuda.synchronize()
        c2, s2 = _quantize(x)
        a, b = torch.empty_like(y4), torch.empty_like(y16)
        P.mx_product(c2, wc, ws, a, count, s2)
        P.mx_product(x, wc, ws, b, count)
        assert torch.equal(c2, xc) and torch.equal(a, y4) and torch.equal(b, y16)


def test_codes_past_4_gib():
    """Weights of more than 2^32 bytes of codes: the last expert's last rows."""
    import paper_2411_01433_amd as P
    E, d_in, d_out = 9, 65536, 16384
    wc = torch.zeros((E, d_out, d_in // 2), dtype=torch.uint8, device="cuda")
    ws = torch.full((E, d_out, d_in // 32), 127, dtype=torch.uint8, device="cuda")
    codes, scales = _mx_matrix((1, 3, d_in), 9)
    wc[-1, -3:], ws[-1, -3:] = torch.from_numpy(codes[0]).cuda(), torch.from_numpy(scales[0]).cuda()
    for rows in (2, 70):
        counts = [0] * 8 + [rows]
        count = torch.tensor(counts, dtype=torch.int32).cuda()
        for act in ("16", "4"):
            if act == "4":
                xc, xs = _mx_matrix((rows, d_in), 10)
                x64 = X.mx_values(xc, xs)
                x, x_scales = torch.from_numpy(xc).cuda(), torch.from_numpy(xs).cuda()
            else:
                g = torch.Generator().manual_seed(11)
                x = torch.randn((rows, d_in), generator=g).bfloat16().cuda()
                x64, x_scales = _f64(x), None
            y = torch.empty((rows, d_out), dtype=torch.bfloat16, device="cuda")
            P.mx_product(x, wc, ws, y, count, x_scales)
            ref, S = X.grouped_product(x64, X.mx_values(codes, scales), [rows], np.zeros((rows, 3)))
            _check(_f64(y[:, -3:]), ref, S, d_in, torch.bfloat16)
            assert not y[:, :-3].any()


def test_binding_refuses():
    import paper_2411_01433_amd as P
    u8 = lambda *s: torch.zeros(s, dtype=torch.uint8, device="cuda")
    v = torch.zeros((4, 64), dtype=torch.float16, device="cuda")
    y = torch.zeros((4, 128), dtype=torch.float16, device="cuda")
    n = torch.zeros(2, dtype=torch.int32, device="cuda")
    wc, ws = u8(2, 128, 32), u8(2, 128, 2)
    for bad in (lambda: P.mx_quantize(v.float(), u8(4, 32), u8(4, 2)),
                lambda: P.mx_quantize(v, u8(4, 31), u8(4, 2)), lambda: P.mx_quantize(v, u8(4, 32), u8(4, 3)),
                lambda: P.mx_quantize(v, u8(4, 32), u8(4, 2), v.bfloat16()),
                lambda: P.mx_product(v, wc, ws, y.float(), n), lambda: P.mx_product(v.bfloat16(), wc, ws, y, n),
                lambda: P.mx_product(v, wc, ws[:1], y, n), lambda: P.mx_product(v, wc, ws, y, n, u8(4, 2)),
                lambda: P.mx_product(u8(4, 32), wc, ws, y, n), lambda: P.mx_product(u8(4, 32), wc, ws, y, n, u8(4, 1))):
        with pytest.raises(ValueError):
            bad()
    odd = torch.zeros((4, 96), dtype=torch.float16, device="cuda")
    with pytest.raises(P.MoeError):
        P.mx_quantize(odd, u8(4, 48), u8(4, 3))
