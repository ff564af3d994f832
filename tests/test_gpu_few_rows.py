"""Grouped products of a decode batch: 1 to 17 rows per expert and 8 on average,
rows of 1088 to 8256 columns, so that the tiles' rows pass through LDS in several
slabs with a remainder; outputs on both sides of the rule that has a block's
waves share its columns.  And scale bytes of 255 in MXFP4 products of either type.

Bounds, against 64 bits: those of the grouped products' tests.  u = 2^-24 is half
a step of fp32, S the sum of the magnitudes of an output's n terms: n 2 u S
element by element, 4 u sqrt(n) of the whole output's norm, and half a step of
the output's type (and half of the smallest subnormal of fp16)."""
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


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _normal(g, shape, dtype, std=1.0):
    return (std * torch.randn(shape, generator=g, device="cuda")).to(dtype)


def _check(got, ref, S, n, dtype):
    err = (got.double() - ref).abs()
    assert bool((err <= HALF[dtype] * ref.abs() + n * 2 * U * S + 2.0 ** -25).all())
    small = 2.0 ** -25 * ref.numel() ** 0.5 if dtype is torch.float16 else 0.0
    assert float(err.norm()) <= (HALF[dtype] + 4 * U * n ** 0.5) * float(ref.norm()) + small


COUNTS = [
    [16, 5, 0, 9, 1, 17, 12, 4],        # 8 rows each: the most that go this way
    [11, 13, 14, 15, 0, 0, 10, 1],
    [6, 7, 2, 3, 8, 29, 0, 5],
]


@TYPES
@pytest.mark.parametrize("d_in", [64, 1088, 4160, 8256])
@pytest.mark.parametrize("d_out", [192, 1216, 1344])
@pytest.mark.parametrize("counts", COUNTS, ids=["most", "full", "mixed"])
def test_decode_batch(counts, d_in, d_out, dtype):
    import paper_2411_01433_amd as P
    n, E = sum(counts), len(counts)
    R = min(n + 2, 8 * E)               # (of the last: two rows behind the experts')
    g = _gen(d_in + d_out)
    x, w = _normal(g, (R, d_in), dtype), _normal(g, (E, d_out, d_in), dtype, 0.05)
    x[n:] = float("nan")
    for e, c in enumerate(counts):
        if c == 0:
            w[e] = float("nan")
    count = torch.tensor(counts, dtype=torch.int32).cuda()
    y = torch.full((R, d_out), 7.0, dtype=dtype, device="cuda")
    P.grouped_product(x, w, y, count)
    for e, (a, c) in enumerate(X.expert_rows(counts, R)):
        if c:
            u, v = x[a:a + c].double(), w[e].double().T
            _check(y[a:a + c], u @ v, u.abs() @ v.abs(), d_in, dtype)
    assert bool((y[n:] == 7.0).all())
    again = torch.empty_like(y)
    P.grouped_product(x, w, again, count)
    assert torch.equal(again[:n], y[:n])


@TYPES
@pytest.mark.parametrize("act", ["16", "4"])
@pytest.mark.parametrize("d_in,d_out", [(320, 192), (4160, 192), (8256, 64)])
@pytest.mark.parametrize("rows", [1, 14, 40, 90])
def test_nan_scales(rows, d_in, d_out, act, dtype):
    """Byte 255 in a row of W, also of a block whose codes are zeros, and in a
    block of x: NaN in the outputs that it enters, no other."""
    import paper_2411_01433_amd as P
    g = _gen(rows)
    u8 = lambda lo, hi, *s: torch.randint(lo, hi, s, generator=g, device="cuda", dtype=torch.uint8)
    codes, scales = u8(0, 256, 1, d_out, d_in // 2), u8(114, 127, 1, d_out, d_in // 32)
    last = d_in // 32 - 1
    scales[0, 40, last], scales[0, 3, 1] = 255, 255
    codes[0, 3, 16:32] = 0
    want = torch.zeros((rows, d_out), dtype=torch.bool, device="cuda")
    want[:, 40] = want[:, 3] = True
    if act == "4":
        x, x_scales = u8(0, 256, rows, d_in // 2), u8(114, 127, rows, d_in // 32)
        if rows > 1:
            x_scales[1, last], x_scales[rows - 1, 0] = 255, 255
            x[rows - 1, :16] = 0
    else:
        x, x_scales = torch.ones((rows, d_in), dtype=dtype, device="cuda"), None
        if rows > 1:
            x[1, d_in - 1] = x[rows - 1, 0] = float("nan")
    if rows > 1:
        want[1] = want[rows - 1] = True
    y = torch.empty((rows, d_out), dtype=dtype, device="cuda")
    P.mx_product(x, codes, scales, y, None, x_scales)
    assert torch.equal(torch.isnan(y), want)
