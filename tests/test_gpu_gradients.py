"""Norm and clipping of gradient lists against the float64 oracle.

Bounds.  Squares of fp32 numbers are summed in 64 bits: the norm is off by its
rounding to fp32 (half a step, u = 2^-24) and next to nothing else.  The factor
c is formed from the rounded norm and rounded (u each), the product is rounded
to fp32 (u) and to the tensor's type (half a step, or half of its smallest
subnormal)."""
import numpy as np
import pytest

from oracle import experts_oracle as X

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

U = 2.0 ** -24
HALF = {torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8, torch.float32: 0.0}
TINY = {torch.float16: 2.0 ** -25, torch.bfloat16: 2.0 ** -134, torch.float32: 2.0 ** -150}
F32, F16, BF16 = torch.float32, torch.float16, torch.bfloat16


@pytest.fixture(scope="module", autouse=True)
def _need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2411_01433_amd as P
    P.lib()
    yield


def _f64(t):
    return t.double().cpu().numpy()


LISTS = [
    [((1,), F32)],
    [((3,), F32), ((0,), F16), ((5, 7), BF16), ((64, 64), F16)],
    [((32768,), F32), ((32769,), F16), ((65535,), BF16), ((4, 8192), F32)],
    [((100003,), F32)],
    [((1 + i % 70,), (F32, F16, BF16)[i % 3]) for i in range(700)],
    [((4, 96, 128), F32), ((4, 128), F32), ((128,), F32), ((4, 96, 128), BF16)],
]


def _make(shapes, seed=0, std=0.1):
    g = torch.Generator().manual_seed(seed + len(shapes))
    return [(std * torch.randn(s, generator=g)).to(t).cuda() for s, t in shapes]


def _check(grads, outs, norm, max_norm, before):
    ref, _ = X.clip([_f64(g) for g in before], max_norm)
    got = float(norm.item())
    assert abs(got - ref) <= 1.001 * U * ref
    for g, o in zip(before, outs):
        want = _f64(g) * min(1.0, max_norm / (ref + 1e-6))
        tol = (3.01 * U + HALF[g.dtype]) * np.abs(want) + TINY[g.dtype]
        assert (np.abs(_f64(o) - want) <= tol).all()


@pytest.mark.parametrize("shapes", LISTS, ids=range(len(LISTS)))
@pytest.mark.parametrize("place", ["in", "out"])
def test_clip(shapes, place):
    import paper_2411_01433_amd as P
    grads = _make(shapes)
    before = [g.clone() for g in grads]
    outs = [torch.full_like(g, 7.0) for g in grads] if place == "out" else None
    norm = torch.zeros(1, device="cuda")
    h = P.MoeGradients(grads, outs)
    h.clip(0.05, norm)
    _check(grads, outs or grads, norm, 0.05, before)
    if outs:
        assert all(torch.equal(a, b) for a, b in zip(grads, before))
    again = torch.zeros(1, device="cuda")
    h2 = P.MoeGradients(before)
    h2.norm(again)
    assert torch.equal(again, norm)  # the same gradients give the same bits
    # a norm below the limit: as they are, bit for bit
    big = torch.zeros(1, device="cuda")
    outs2 = [torch.full_like(g, 7.0) for g in before] if place == "out" else None
    kept = [g.clone() for g in before]
    h3 = P.MoeGradients(before, outs2)
    h3.clip(1e6, big)
    assert all(torch.equal(a, b) for a, b in zip(outs2 or before, kept))
    for x in (h, h2, h3):
        x.destroy()


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
def test_views_at_every_offset(dtype):
    """Tensors that start and end off the 16-byte grid, in and out at offsets of
    their own; what lies around them stays as it is."""
    import paper_2411_01433_amd as P
    g = torch.Generator().manual_seed(3)
    flat = (0.1 * torch.randn(40000, generator=g)).to(dtype).cuda()
    to = torch.full((40000,), 7.0, dtype=dtype, device="cuda")
    at, ins, outs, where = 1, [], [], []
    for k, n in enumerate((1, 2, 7, 8, 9, 15, 16, 17, 100, 1000, 33000)):
        o = at + k % 5
        ins.append(flat[at:at + n])
        outs.append(to[o:o + n])
        where.append((o, n))
        at += n + 7
    h, norm = P.MoeGradients(ins, outs), torch.zeros(1, device="cuda")
    h.clip(0.01, norm)
    _check(ins, outs, norm, 0.01, [t.clone() for t in ins])
    hole = torch.ones(40000, dtype=torch.bool)
    for o, n in where:
        hole[o:o + n] = False
    assert (to.cpu()[hole] == 7.0).all()
    before = flat.clone()
    P.MoeGradients(ins).clip(0.01, norm)
    hole = torch.ones(40000, dtype=torch.bool)
    for t in ins:
        a = t.storage_offset()
        hole[a:a + t.numel()] = False
    assert torch.equal(flat.cpu()[hole], before.cpu()[hole])
    assert all(torch.equal(a, b) for a, b in zip(ins, outs))


@pytest.mark.parametrize("size", [1e30, 1e-30, 2.0 ** -149])
def test_sizes_whose_squares_leave_fp32(size):
    import paper_2411_01433_amd as P
    grads = [torch.full((1000,), size, device="cuda"), torch.zeros(7, device="cuda")]
    before = [g.clone() for g in grads]
    norm = torch.zeros(1, device="cuda")
    P.MoeGradients(grads).clip(1.0, norm)
    ref, _ = X.clip([_f64(g) for g in before], 1.0)
    # (half of the smallest subnormal where the norm is one)
    assert abs(float(norm.item()) - ref) <= 1.001 * U * ref + 2.0 ** -150
    if size > 1:
        _check(grads, grads, norm, 1.0, before)
    else:
        assert torch.equal(grads[0], before[0])


@pytest.mark.parametrize("bad", [float("inf"), float("nan"), float("-inf")])
@pytest.mark.parametrize("place", ["in", "out"])
def test_not_finite(bad, place):
    """The norm shows it and nothing is scaled."""
    import paper_2411_01433_amd as P
    grads = [torch.ones(50000, device="cuda"), torch.ones(9, dtype=F16, device="cuda")]
    grads[0][40000] = bad
    before = [g.clone() for g in grads]
    outs = [torch.zeros_like(g) for g in grads] if place == "out" else None
    norm = torch.zeros(1, device="cuda")
    P.MoeGradients(grads, outs).clip(0.1, norm)
    assert not torch.isfinite(norm).any()
    for a, b in zip(outs or grads, before):
        assert torch.equal(a.view(torch.int16 if a.dtype is F16 else torch.int32),
                           b.view(torch.int16 if b.dtype is F16 else torch.int32))


def test_norm_beyond_fp32_is_infinite():
    import paper_2411_01433_amd as P
    g = torch.full((64,), 3e38, device="cuda")
    norm = torch.zeros(1, device="cuda")
    P.MoeGradients([g]).clip(1.0, norm)
    assert norm.item() == float("inf") and (g == 3e38).all()


def test_scale_by_a_norm_joined_elsewhere():
    """The norm of two lists, joined by the caller, scales both."""
    import paper_2411_01433_amd as P
    a, b = _make(LISTS[5]), _make(LISTS[2], 9)
    before = [g.clone() for g in a + b]
    ha, hb = P.MoeGradients(a), P.MoeGradients(b)
    n = torch.zeros(2, device="cuda")
    ha.norm(n[:1]), hb.norm(n[1:])
    total = n.double().square().sum().sqrt().float().view(1)
    ha.scale(0.5, total), hb.scale(0.5, total)
    # the joined norm carries the two roundings and its own
    ref, _ = X.clip([_f64(g) for g in before], 0.5)
    assert abs(total.item() - ref) <= 2.001 * U * ref
    for g, o in zip(before, a + b):
        want = _f64(g) * (0.5 / (ref + 1e-6))
        assert (np.abs(_f64(o) - want) <= (5 * U + HALF[g.dtype]) * np.abs(want) + TINY[g.dtype]).all()


def test_nothing_to_clip():
    import paper_2411_01433_amd as P
    norm = torch.full((1,), 7.0, device="cuda")
    P.MoeGradients([torch.empty(0, device="cuda"), torch.empty((0, 5), dtype=F16, device="cuda")]).clip(1.0, norm)
    assert norm.item() == 0.0


def test_captured_and_on_another_stream():
    import paper_2411_01433_amd as P
    grads = _make(LISTS[4]) + _make(LISTS[2], 1)
    outs = [torch.empty_like(g) for g in grads]
    outs2 = [torch.empty_like(g) for g in grads]
    h, h2 = P.MoeGradients(grads, outs), P.MoeGradients(grads, outs2)
    n1, n2 = torch.zeros(1, device="cuda"), torch.zeros(1, device="cuda")
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        h.clip(0.5, n1)
    side = torch.cuda.Stream()
    for k in range(4):
        for g in grads:
            g.mul_(1.0 + 0.3 * k)
        graph.replay()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            h2.clip(0.5, n2)
        torch.cuda.synchronize()
        assert torch.equal(n1, n2) and all(torch.equal(a, b) for a, b in zip(outs, outs2))
        _check(grads, outs, n1, 0.5, grads)


def test_past_4_gib():
    import paper_2411_01433_amd as P
    g = torch.zeros((1 << 32) + 5, dtype=F16, device="cuda")
    g[-3:] = torch.tensor([3.0, 4.0, 12.0], dtype=F16)
    norm = torch.zeros(1, device="cuda")
    P.MoeGradients([g]).clip(6.5, norm)
    assert norm.item() == 13.0
    assert g[-3:].tolist() == [1.5, 2.0, 6.0] and not g[:-3].any()


def test_refusals():
    import paper_2411_01433_amd as P
    g = torch.zeros(8, device="cuda")
    n = torch.zeros(1, device="cuda")
    for bad in (lambda: P.MoeGradients([g.cpu()]), lambda: P.MoeGradients([g.double()]),
                lambda: P.MoeGradients([g.view(2, 4).t()]), lambda: P.MoeGradients([g], [g[:4]]),
                lambda: P.MoeGradients([g], [g.half()]), lambda: P.MoeGradients([g], []),
                lambda: P.MoeGradients([g]).clip(1.0, n.double())):
        with pytest.raises(ValueError):
            bad()
    for bad in (lambda: P.MoeGradients([]), lambda: P.MoeGradients([g, g]),
                lambda: P.MoeGradients([g[:5], g[4:]]), lambda: P.MoeGradients([g]).clip(0.0, n),
                lambda: P.MoeGradients([g]).clip(float("nan"), n),
                lambda: P.MoeGradients([g]).scale(float("inf"), n)):
        with pytest.raises(P.MoeError):
            bad()
    h = P.MoeGradients([g])
    h.destroy()
    with pytest.raises(P.MoeError):
        h.clip(1.0, n)
