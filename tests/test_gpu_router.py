"""Routing rules and their backward pass against the float64 oracle.

Selected experts and their counts are equal, near scores included (both sides
go by 64-bit sums).  Bounds of the numbers, u = 2^-24:
 * a logit is a sum of d exact products: at most d/32 + 64 roundings of 2u of
   the sum of their magnitudes lie on any element's way;
 * a weight is a ratio of exponentials: twice the largest error of its logits,
   and 64 u (1 + the largest |logit|) for the functions and their arguments;
 * a logit's gradient: 64 u (1 + max |logit|) of its terms' magnitudes, and
   2^-22 of itself (held in two numbers of 16 bits at least) and 2^-38 of the
   call's largest (below what those can hold);
 * its products: as the logits', over experts or tokens."""
import numpy as np
import pytest

from oracle import routing_oracle as R

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

U = 2.0 ** -24
HALF = {torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}
F16, BF16 = torch.float16, torch.bfloat16


@pytest.fixture(scope="module", autouse=True)
def _need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2411_01433_amd as P
    P.lib()
    yield


def _np(t):
    return None if t is None else t.double().cpu().numpy() if t.is_floating_point() else t.cpu().numpy()


def make(rule, wg, bias, T, backward=False):
    import paper_2411_01433_amd as P
    E, d = wg.shape
    return P.MoeRouter(d, E, rule.top_k, T, wg, bias, dtype=wg.dtype, score=rule.score,
                       n_groups=rule.n_groups, top_groups=rule.top_groups,
                       group_best=rule.group_best, renormalize=rule.renormalize,
                       scale=rule.scale, backward=backward)


def inputs(T, d, E, dtype, seed, bias):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn((T, d), generator=g).to(dtype).cuda()
    wg = (torch.randn((E, d), generator=g) * d ** -0.5 * 1.3).to(dtype).cuda()
    b = (torch.randn(E, generator=g) * bias).cuda() if bias else None
    return x, wg, b, g


def outs(T, K, E):
    """Buffers of one call, one row longer than the call: what is behind the
    last token stays as it is."""
    return (torch.full((T + 1, K), -7, dtype=torch.int32, device="cuda"),
            torch.full((T + 1, K), -7.0, device="cuda"),
            torch.full((T + 1, E), -7.0, device="cuda"),
            torch.full((E,), -7, dtype=torch.int32, device="cuda"))


def logit_bound(x, wg):
    x, wg = np.abs(_np(x)), np.abs(_np(wg))
    return (x.shape[1] / 32 + 64) * 2 * U * (x @ wg.T)


def check(rule, x, wg, bias, r=None):
    """One call of the library against the oracle; returns its outputs."""
    T, K, E = x.shape[0], rule.top_k, wg.shape[0]
    own = r is None
    r = r or make(rule, wg, bias, T)
    idx, w, lg, count = outs(T, K, E)
    r.route(x, idx[:T], w[:T], lg[:T], count)
    torch.cuda.synchronize()
    ref_idx, ref_w, ref_l, ref_count = R.route(rule, _np(x), _np(wg), _np(bias))
    assert np.array_equal(_np(idx[:T]), ref_idx), np.argwhere(_np(idx[:T]) != ref_idx)[:4]
    assert np.array_equal(_np(count), ref_count)
    fin = np.isfinite(ref_l)
    off = np.abs(np.where(fin, _np(lg[:T]) - np.where(fin, ref_l, 0), 0))
    bound = np.where(fin, logit_bound(x, wg), np.inf) + U * np.abs(np.where(fin, ref_l, 0))
    assert (off <= bound).all(), (off / bound).max()
    big = np.where(fin, np.abs(ref_l), 0).max(-1, keepdims=True)
    err = np.where(fin, bound, 0).max(-1, keepdims=True)
    tol = (2 * err + 64 * U * (1 + big)) * np.abs(ref_w) + 1e-37
    assert (np.abs(_np(w[:T]) - ref_w) <= tol).all(), (np.abs(_np(w[:T]) - ref_w) / tol).max()
    assert (idx[T] == -7).all() and (w[T] == -7).all() and (lg[T] == -7).all()
    # without the optional outputs, the same
    idx2, w2 = torch.empty_like(idx[:T]), torch.empty_like(w[:T])
    r.route(x, idx2, w2)
    assert torch.equal(idx2, idx[:T]) and torch.equal(w2, w[:T])
    if own:
        r.destroy()
    return idx[:T], w[:T], lg[:T]


S, G = R.SOFTMAX, R.SIGMOID
CASES = [
    # T, d, E, type, bias, rule
    (1, 4096, 16, F16, 0, R.Rule(2)),
    (1, 64, 1, F16, 0, R.Rule(1)),
    (1, 16384, 8, BF16, 0, R.Rule(2, renormalize=False)),
    (2, 128, 2, F16, 0.1, R.Rule(2, score=G, renormalize=False)),
    (3, 320, 6, BF16, 0, R.Rule(3, score=G, scale=2.5)),
    (5, 1024, 17, F16, 0.02, R.Rule(4, score=G)),
    (8, 4096, 256, F16, 0.02, R.Rule(8, score=G, n_groups=8, top_groups=4, group_best=2, scale=2.5)),
    (17, 2048, 60, F16, 0, R.Rule(4, renormalize=False)),
    (33, 192, 160, F16, 0, R.Rule(6, n_groups=8, top_groups=3, renormalize=False, scale=16.0)),
    (64, 512, 65, BF16, 0.001, R.Rule(8, renormalize=True)),
    (65, 320, 64, F16, 0.02, R.Rule(8, score=G, n_groups=64, top_groups=16, group_best=2)),
    (130, 256, 96, BF16, 0.01, R.Rule(5, n_groups=4, top_groups=2, group_best=2)),
    (200, 128, 512, F16, 0.02, R.Rule(16, score=G, n_groups=16, top_groups=4, group_best=2)),
    (257, 1088, 128, F16, 0, R.Rule(1, score=G, renormalize=False)),
    (515, 64, 511, F16, 0, R.Rule(16)),
    (600, 2048, 256, BF16, 0.02, R.Rule(8, score=G, n_groups=8, top_groups=4, group_best=1)),
    (1100, 256, 8, F16, 0, R.Rule(2)),
    (2100, 128, 40, F16, 0.002, R.Rule(4, renormalize=False)),
    (3000, 512, 256, F16, 0.0008, R.Rule(8, renormalize=False)),
    # every kind of selection kernel at every number of experts per lane, and
    # groups whose number or size is no power of two
    (256, 128, 40, F16, 0.02, R.Rule(5, score=G, n_groups=5, top_groups=2, group_best=2)),
    (700, 64, 96, F16, 0, R.Rule(6, n_groups=12, top_groups=5, group_best=2)),
    (2300, 128, 100, BF16, 0.02, R.Rule(7, score=G, n_groups=20, top_groups=6, group_best=2)),
    (2500, 64, 512, F16, 0.02, R.Rule(16, score=G, n_groups=32, top_groups=9, group_best=2)),
    (5000, 64, 13, F16, 0, R.Rule(13, renormalize=False)),
    (5001, 128, 16, BF16, 0.02, R.Rule(16, score=G, n_groups=16, top_groups=16)),
    (4100, 256, 60, F16, 0.02, R.Rule(4, score=G, n_groups=3, top_groups=1)),
]


@pytest.mark.parametrize("T,d,E,dtype,bias,rule", CASES,
                         ids=[f"t{c[0]}_d{c[1]}_e{c[2]}" for c in CASES])
def test_forward(T, d, E, dtype, bias, rule):
    x, wg, b, _ = inputs(T, d, E, dtype, T * 131 + d + E, bias)
    check(rule, x, wg, b)


@pytest.mark.parametrize("rule", [
    R.Rule(4), R.Rule(4, score=G, n_groups=4, top_groups=2, group_best=2),
    R.Rule(4, renormalize=False, n_groups=4, top_groups=2)], ids=["softmax", "sigmoid", "groups"])
@pytest.mark.parametrize("bias", [False, True])
def test_ties_go_to_the_lower_index(rule, bias):
    """Equal gate rows, zero tokens and integers whose sums are exact: ties of
    experts and of groups everywhere."""
    g = torch.Generator().manual_seed(4)
    x = torch.randint(-2, 3, (40, 128), generator=g).half()
    x[3] = 0
    wg = torch.randint(-1, 2, (16, 128), generator=g).half() / 16
    wg[8:] = wg[:8]
    wg[5] = wg[2]
    b = torch.zeros(16) if bias else None
    check(rule, x.cuda(), wg.cuda(), None if b is None else b.cuda())


def test_near_ties_go_by_the_exact_sums():
    """Gate rows that differ by one step in one element, beside large terms that
    cancel: fp32 sums cannot tell them apart, 64-bit ones do."""
    g = torch.Generator().manual_seed(11)
    d, E, T = 1024, 32, 64
    base = torch.randn(d, generator=g)
    wg = base.repeat(E, 1).half()
    for e in range(E):
        j = int(torch.randint(0, d, (1,), generator=g))
        bits = wg[e].view(torch.int16)
        bits[j] += 1 if e % 2 else -1
    x = (torch.randn((T, d), generator=g) * 30).half()
    for rule, bias in ((R.Rule(8), None), (R.Rule(8, score=G), torch.zeros(E)),
                       (R.Rule(8, n_groups=4, top_groups=2, group_best=2), torch.zeros(E))):
        # (scores that saturate tie, so the logits are kept small)
        xs = x if bias is None else x / 256
        check(rule, xs.half().cuda(), wg.cuda(), None if bias is None else bias.cuda())


@pytest.mark.parametrize("dtype,x_scale,w_scale", [
    (F16, 2.0 ** -24, 1.0), (F16, 2.0 ** -24, 2.0 ** -20), (BF16, 1e-25, 1.0), (BF16, 1e15, 1e12),
    (F16, 1024.0, 64.0)], ids=["f16_subnormal", "f16_both_subnormal", "bf16_tiny", "bf16_huge", "f16_large"])
@pytest.mark.parametrize("E", [12, 40])
def test_near_ties_at_the_ends_of_the_range(dtype, x_scale, w_scale, E):
    """Products and squares near the ends of the types: the bound of the sums'
    errors holds there too.  Integers times powers of two and a gate whose rows
    differ in one place, so that many sums are near or equal."""
    g = torch.Generator().manual_seed(13)
    d, T = 192, 40
    x = torch.randint(-7, 8, (T, d), generator=g).float() * x_scale
    wg = torch.randint(-3, 4, (d,), generator=g).float().repeat(E, 1)
    wg[torch.arange(E), torch.randint(0, d, (E,), generator=g)] += 1
    wg *= w_scale
    x, wg = x.to(dtype).cuda(), wg.to(dtype).cuda()
    check(R.Rule(4), x, wg, None)
    if x_scale < 1:
        b = (torch.randn(E, generator=g) * 0.1).cuda()
        check(R.Rule(4, score=G), x, wg, b)
        check(R.Rule(4, renormalize=False), x, wg, b)


def test_rows_of_zeros_in_a_long_call():
    """A padded batch: tokens of zeros tie everywhere, by index."""
    T, d, E = 2600, 128, 96
    x, wg, _, _ = inputs(T, d, E, F16, 3, 0)
    x[1000:2200] = 0
    for bias in (None, torch.zeros(E, device="cuda")):
        idx, _, _ = check(R.Rule(6, score=G, n_groups=8, top_groups=4, group_best=2), x, wg, bias)
        assert (idx[1000:2200].cpu() == torch.arange(6)).all()
    wg.zero_()   # and a gate that has not learnt anything yet
    check(R.Rule(6, score=G), x, wg, torch.zeros(E, device="cuda"))


def test_masked_experts_and_rows_without_any():
    """Bias -inf masks experts, whole groups, all but one, all; logits that are
    not finite (tokens with infinities and NaN) take no part."""
    T, d, E = 24, 256, 32
    x, wg, _, g = inputs(T, d, E, F16, 21, 0)
    x[5] = float("nan")
    x[6, 3] = float("inf")
    x[7] = 0
    b = (torch.randn(E, generator=g) * 0.02).cuda()
    b[4:12] = -float("inf")
    b[20] = float("nan")
    b[21] = float("inf")
    rule = R.Rule(6, score=G, n_groups=8, top_groups=2, group_best=2)
    idx, w, _ = check(rule, x, wg, b)
    assert (idx[5] == -1).all() and (w[5] == 0).all()
    check(R.Rule(6), x, wg, b)
    one = torch.full((E,), -float("inf"), device="cuda")
    one[9] = 0.0
    for rule in (R.Rule(3), R.Rule(3, score=G, n_groups=4, top_groups=4),
                 R.Rule(3, renormalize=False, n_groups=8, top_groups=1, group_best=2)):
        idx, _, _ = check(rule, x, wg, one)
        assert (idx[0].cpu() == torch.tensor([9, -1, -1])).all()
        one2 = torch.full((E,), -float("inf"), device="cuda")
        idx, w, _ = check(rule, x, wg, one2)
        assert (idx == -1).all() and (w == 0).all()


@pytest.mark.parametrize("T", [5, 300, 2100])
@pytest.mark.parametrize("E,G,keep", [(16, 4, 2), (64, 8, 3), (300, 10, 4)])
def test_masks_of_the_lowest_value(T, E, G, keep):
    """A bias of fp32's lowest value is finite: such experts come after all
    others, by index, and groups of them before groups of experts at -inf,
    though two of them add up to no fp32 number.  And of its largest value."""
    x, wg, _, g = inputs(T, 128, E, F16, 23, 0)
    lowest, size = torch.finfo(torch.float32).min, E // G
    b = torch.randn(E, generator=g) * 0.02
    b[torch.randperm(E, generator=g)[:E // 3]] = lowest
    for score in (R.SIGMOID, R.SOFTMAX):
        check(R.Rule(4, score=score, n_groups=G, top_groups=keep, group_best=2), x, wg, b.cuda())
        check(R.Rule(4, score=score), x, wg, b.cuda())
    rule = R.Rule(min(size + 1, 16), score=R.SIGMOID, n_groups=G, top_groups=2, group_best=2)
    only = torch.full((E,), -float("inf"))   # all groups masked, one by the lowest value
    only[size * (G - 1):] = lowest
    only[3] = 0.0
    idx, _, _ = check(rule, x, wg, only.cuda())
    assert (idx[:, 1].cpu() == size * (G - 1)).all()
    top = torch.zeros(E)
    top[2 * size:] = -lowest
    check(rule, x, wg, top.cuda())


@pytest.mark.parametrize("score", [R.SIGMOID, R.SOFTMAX])
@pytest.mark.parametrize("T", [1, 300, 2100])
def test_biases_that_cancel_the_scores(T, score):
    """Keys that are all within fp32's rounding of zero, of scores that differ:
    every comparison takes the sums, and a softmax's denominator, in 64 bits."""
    d, E = 192, 40
    for seed in range(8):
        x, wg, _, _ = inputs(T, d, E, F16, 100 + seed, 0)
        x[:] = x[0]
        l = _np(x[:1]) @ _np(wg).T
        b = torch.from_numpy(-R.scores(R.Rule(4, score=score), l[0])).float().cuda()
        check(R.Rule(4, score=score, n_groups=10, top_groups=3, group_best=2), x, wg, b)
        check(R.Rule(6, score=score, n_groups=4, top_groups=2), x, wg, b)
        check(R.Rule(4, score=score), x, wg, b)


def test_far_logits():
    """Scores that saturate or underflow: shares by their logarithms."""
    T, d, E = 16, 128, 12
    x, wg, _, _ = inputs(T, d, E, BF16, 5, 0)
    for f in (30.0, 300.0):
        for rule in (R.Rule(4), R.Rule(4, score=G), R.Rule(4, renormalize=False),
                     R.Rule(4, score=G, renormalize=False)):
            check(rule, (x * f).to(BF16), wg, None)


def test_bias_and_gate_updated_in_place():
    T, d, E = 50, 256, 24
    x, wg, b, _ = inputs(T, d, E, F16, 9, 0.02)
    rule = R.Rule(4, score=G)
    r = make(rule, wg, b, T)
    for _ in range(3):
        check(rule, x, wg, b, r)
        b.neg_()
        wg.mul_(0.5)
    # fewer tokens than the handle takes, on the same handle
    check(rule, x[:7].contiguous(), wg, b, r)
    r.destroy()


# ---- backward -------------------------------------------------------------------

def gradient_bounds(rule, l, idx, dw, dl, g):
    """Bound of the logits' gradient [T, E]."""
    l, T, E = np.asarray(l, np.float64), l.shape[0], l.shape[1]
    part = np.zeros((T, E))
    for t in range(T):
        on = [k for k in range(rule.top_k) if 0 <= idx[t, k] < E and np.isfinite(l[t, idx[t, k]])]
        if not on:
            continue
        ids = idx[t, on]
        up = rule.scale * np.abs(dw[t, on]).max()
        if rule.renormalize:
            np.add.at(part[t], ids, 2 * up * R.shares(rule, l[t], ids))
        elif rule.score == G:
            np.add.at(part[t], ids, up * R.scores(rule, l[t])[ids])
        else:
            s = R.scores(rule, l[t])
            np.add.at(part[t], ids, up * s[ids])
            part[t] += s * up * rule.top_k
    big = np.where(np.isfinite(l), np.abs(l), 0).max(-1, keepdims=True)
    own = 0 if dl is None else np.abs(dl)
    return (64 * U * (1 + big) * part + 2 * U * own + 2.0 ** -22 * np.abs(g)
            + 2.0 ** -38 * np.abs(g).max())


def check_backward(rule, x, wg, logits, idx, dw, dl, r=None):
    T, d, E = x.shape[0], x.shape[1], wg.shape[0]
    own = r is None
    r = r or make(rule, wg, None, T, backward=True)
    dx = torch.full((T + 1, d), 7.0, dtype=x.dtype, device="cuda")
    dwg = torch.empty((E, d), device="cuda")
    r.backward(x, logits, idx, dw, dx[:T], dwg, dl)
    torch.cuda.synchronize()
    rx, rw, g = R.route_backward(rule, _np(x), _np(wg), _np(logits), _np(idx), _np(dw), _np(dl))
    eg = gradient_bounds(rule, _np(logits), _np(idx), _np(dw), _np(dl), g)
    ax, aw = np.abs(_np(x)), np.abs(_np(wg))
    tol = (HALF[x.dtype] * np.abs(rx) + eg @ aw + (E / 16 + 32) * 2 * U * (np.abs(g) @ aw) + 2.0 ** -25)
    off = np.abs(_np(dx[:T]) - rx)
    assert (off <= tol).all(), ("d_x", (off / tol).max())
    tol = eg.T @ ax + (128 + T / 256) * 2 * U * (np.abs(g).T @ ax)
    off = np.abs(_np(dwg) - rw)
    assert (off <= tol).all(), ("d_w_router", (off / np.maximum(tol, 1e-300)).max())
    assert (dx[T] == 7.0).all()
    # the same bits again; each output alone
    dx2, dwg2 = torch.empty_like(dx[:T]), torch.empty_like(dwg)
    r.backward(x, logits, idx, dw, dx2, None, dl)
    r.backward(x, logits, idx, dw, None, dwg2, dl)
    assert torch.equal(dx2, dx[:T]) and torch.equal(dwg2, dwg)
    if own:
        r.destroy()
    return dx[:T], dwg


BACK = [
    # T, d, E, type, rule, gradient of the logits too
    (1, 64, 1, F16, R.Rule(1), True),
    (1, 4096, 16, F16, R.Rule(2), False),
    (3, 320, 6, BF16, R.Rule(3, score=G, renormalize=False, scale=2.5), True),
    (17, 128, 17, F16, R.Rule(4, renormalize=False), False),
    (64, 512, 256, F16, R.Rule(8, score=G, scale=2.5), False),
    (65, 192, 60, BF16, R.Rule(4, renormalize=False), True),
    (127, 1088, 96, F16, R.Rule(5, score=G), True),
    (300, 256, 160, BF16, R.Rule(6), False),
    (513, 320, 512, F16, R.Rule(16, renormalize=False, scale=16.0), True),
    (1025, 2048, 8, F16, R.Rule(2), False),
    (3000, 256, 64, F16, R.Rule(4, score=G, renormalize=False), True),
    (2049, 1024, 130, BF16, R.Rule(8, score=G), False),
    (2, 16384, 40, F16, R.Rule(4), True),
]


def grads(T, K, E, g, dl):
    return (torch.randn((T, K), generator=g).cuda(),
            (0.01 * torch.randn((T, E), generator=g)).cuda() if dl else None)


@pytest.mark.parametrize("T,d,E,dtype,rule,dl", BACK, ids=[f"t{c[0]}_d{c[1]}_e{c[2]}" for c in BACK])
def test_backward(T, d, E, dtype, rule, dl):
    x, wg, _, g = inputs(T, d, E, dtype, T * 7 + d + E, 0)
    idx, _, l, _ = R.route(rule, _np(x), _np(wg))
    dw, dl = grads(T, rule.top_k, E, g, dl)
    check_backward(rule, x, wg, torch.from_numpy(l).float().cuda(), torch.from_numpy(idx).cuda(), dw, dl)


@pytest.mark.parametrize("rule", [R.Rule(4), R.Rule(4, score=G), R.Rule(4, renormalize=False),
                                  R.Rule(4, score=G, renormalize=False)],
                         ids=["softmax", "sigmoid", "softmax_all", "sigmoid_raw"])
def test_backward_of_odd_slots(rule):
    """Empty slots, indices out of range, the same index twice, logits that are
    not finite, gradients of very different sizes, rows of zeros."""
    T, d, E = 70, 192, 24
    x, wg, _, g = inputs(T, d, E, F16, 77, 0)
    idx, _, l, _ = R.route(rule, _np(x), _np(wg))
    idx[0] = -1
    idx[1, 2:] = -1
    idx[2, 1] = idx[2, 0]
    idx[3] = idx[3, 0]
    idx[4, 0], idx[4, 1] = E, -2 ** 31
    idx[5, 3] = 2 ** 31 - 1
    l[6, idx[6, 0]] = np.nan
    l[7, :] = np.inf
    l[8, idx[8, 1]] = -np.inf
    dw, dl = grads(T, rule.top_k, E, g, True)
    dw[10:20] *= 1e-6
    dw[20:30] *= 1e4
    dl[10:30] = 0
    dw[30:40] = 0
    dl[30:40] = 0
    check_backward(rule, x, wg, torch.from_numpy(l).float().cuda(), torch.from_numpy(idx).cuda(), dw, dl)
    check_backward(rule, x, wg, torch.from_numpy(l).float().cuda(), torch.from_numpy(idx).cuda(), dw, None)


def test_backward_against_differences():
    """<gradient, direction> of both inputs against central differences of the
    64-bit forward pass along that direction."""
    T, d, E = 40, 128, 20
    rule = R.Rule(4, score=G, scale=2.5)
    x, wg, _, g = inputs(T, d, E, F16, 8, 0)
    idx, _, l, _ = R.route(rule, _np(x), _np(wg))
    dw, dl = grads(T, 4, E, g, True)
    dx, dwg = check_backward(rule, x, wg, torch.from_numpy(l).float().cuda(),
                             torch.from_numpy(idx).cuda(), dw, dl)

    def loss(xv, wv):
        l = xv @ wv.T
        return sum((R.weights(rule, l[t], idx[t]) * _np(dw)[t]).sum() for t in range(T)) + (l * _np(dl)).sum()

    rng = np.random.default_rng(3)
    vx, vw = rng.normal(size=x.shape), rng.normal(size=wg.shape)
    h, x64, w64 = 1e-6, _np(x), _np(wg)
    num = (loss(x64 + h * vx, w64) - loss(x64 - h * vx, w64)) / (2 * h)
    # each element of d_x is half a step off at most, signs of vx are random
    assert abs(num - (_np(dx) * vx).sum()) <= 2.0 ** -11 * np.abs(_np(dx) * vx).sum()
    num = (loss(x64, w64 + h * vw) - loss(x64, w64 - h * vw)) / (2 * h)
    assert abs(num - (_np(dwg) * vw).sum()) <= 1e-6 * np.abs(_np(dwg) * vw).sum() + 1e-6 * abs(num)


# ---- handles, streams, graphs -----------------------------------------------------

def test_refusals():
    import paper_2411_01433_amd as P
    T, d, E = 8, 128, 6
    x, wg, b, _ = inputs(T, d, E, F16, 1, 0.1)
    r = make(R.Rule(2), wg, b, T)
    idx, w, lg, count = outs(T - 1, 2, E)
    with pytest.raises(P.MoeError, match="n_tokens"):
        r.route(torch.zeros((T + 1, d), dtype=F16, device="cuda"),
                torch.zeros((T + 1, 2), dtype=torch.int32, device="cuda"),
                torch.zeros((T + 1, 2), device="cuda"))
    with pytest.raises(P.MoeError, match="n_tokens"):
        r.route(x[:0], idx[:0], w[:0])
    with pytest.raises(P.MoeError, match="NULL"):
        r.route(x, None, w)
    for bad in (dict(x=x.bfloat16()), dict(x=x[:, :64].contiguous()), dict(x=x.t()),
                dict(topk_idx=idx.long()), dict(topk_w=w[:4]), dict(logits=lg[:, :3]),
                dict(expert_count=count.float())):
        with pytest.raises(ValueError):
            r.route(**{**dict(x=x, topk_idx=idx, topk_w=w), **bad})
    with pytest.raises(P.MoeError, match="aligned"):
        r.route(torch.zeros(T * d + 4, dtype=F16, device="cuda")[4:].view(T, d), idx, w)
    with pytest.raises(P.MoeError, match="MOE_ROUTER_BACKWARD"):
        r.backward(x, lg, idx, w, x)
    rb = make(R.Rule(2), wg, b, T, backward=True)
    with pytest.raises(P.MoeError, match="both NULL"):
        rb.backward(x, lg, idx, w)
    with pytest.raises(P.MoeError, match="NULL"):
        rb.backward(x, None, idx, w, x)
    with pytest.raises(ValueError):
        rb.backward(x, lg, idx, w, x.float())
    with pytest.raises(ValueError):
        rb.backward(x, lg, idx, w, x, torch.zeros((E, d), dtype=F16, device="cuda"))
    rb.destroy()
    r.destroy()
    with pytest.raises(P.MoeError):
        r.route(x, idx, w)


def test_offsets_past_31_bits():
    """The largest call, 2 GiB of tokens: its last 64 as in a call of their own."""
    T, d, E, n = 65536, 16384, 20, 64
    rule = R.Rule(4, score=G, n_groups=5, top_groups=3, group_best=2)
    g = torch.Generator(device="cuda").manual_seed(4)
    x = torch.randn((T, d), generator=g, device="cuda", dtype=F16)
    wg = torch.randn((E, d), generator=g, device="cuda").mul_(d ** -0.5).to(F16)
    b = torch.randn(E, generator=g, device="cuda") * 0.02
    tail = x[-n:].clone()
    own, _, lg2 = check(rule, tail, wg, b)
    r = make(rule, wg, b, T, backward=True)
    idx, w, lg = (torch.empty((T, k), dtype=t, device="cuda")
                  for k, t in ((4, torch.int32), (4, torch.float32), (E, torch.float32)))
    count = torch.empty(E, dtype=torch.int32, device="cuda")
    r.route(x, idx, w, lg, count)
    assert torch.equal(idx[-n:], own[:n])
    assert torch.equal(count.long(), torch.bincount(idx.flatten().long(), minlength=E))
    assert (np.abs(_np(lg[-n:]) - _np(tail) @ _np(wg).T) <= logit_bound(tail, wg)).all()
    # gradients of the last 64 weights only: the others add zeros
    up = torch.zeros((T, 4), device="cuda")
    up[-n:] = torch.randn((n, 4), generator=g, device="cuda")
    dx, dw = torch.empty_like(x), torch.empty((E, d), device="cuda")
    r.backward(x, lg, idx, up, dx, dw)
    dx2, dw2 = torch.empty_like(tail), torch.empty((E, d), device="cuda")
    r.backward(tail, lg[-n:].clone(), idx[-n:].clone(), up[-n:].clone(), dx2, dw2)
    assert torch.equal(dx[-n:], dx2) and torch.equal(dw, dw2)
    assert not dx[:-n].any()
    r.destroy()


def test_tensors_of_another_device_are_refused(monkeypatch):
    import paper_2411_01433_amd as P
    x, wg, _, _ = inputs(4, 128, 6, F16, 1, 0)
    r = make(R.Rule(2), wg, None, 4, backward=True)
    idx, w, lg, _ = outs(3, 2, 6)
    h = torch.zeros((4, 128), device="cuda")
    with monkeypatch.context() as m:
        m.setattr(torch.cuda, "current_device", lambda: 1)
        with pytest.raises(ValueError, match="current device"):
            P.layernorm(h, x)
        with pytest.raises(ValueError, match="current device"):
            P.layernorm_backward(x, h, h)
    r._device = 1
    with pytest.raises(ValueError, match="on device 1"):
        r.route(x, idx, w)
    with pytest.raises(ValueError, match="on device 1"):
        r.backward(x, lg, idx, w, x)
    r._device = 0
    r.destroy()


def test_two_handles_on_two_streams():
    """Handles own their workspaces: two of them run side by side."""
    T, d, E = 400, 512, 64
    rule = R.Rule(4, score=G)
    x, wg, b, g = inputs(T, d, E, F16, 2, 0.02)
    x2 = torch.randn((T, d), generator=g).half().cuda()
    ref = [check(rule, v, wg, b)[:2] for v in (x, x2)]
    hs = [make(rule, wg, b, T) for _ in range(2)]
    ss = [torch.cuda.Stream() for _ in range(2)]
    out = [outs(T - 1, 4, E) for _ in range(2)]
    torch.cuda.synchronize()
    for _ in range(20):
        for r, s, v, o in zip(hs, ss, (x, x2), out):
            r.route(v, o[0], o[1], o[2], o[3], stream=s)
    torch.cuda.synchronize()
    for o, (idx, w) in zip(out, ref):
        assert torch.equal(o[0], idx) and torch.equal(o[1], w)
    for r in hs:
        r.destroy()


@pytest.mark.parametrize("T,E", [(1, 16), (300, 96)])
def test_captured_pass(T, E):
    """Forward and backward captured into two graphs of one handle, replayed in
    turn between eager passes on changing inputs: the eager bits every time."""
    d, K = 512, 4
    rule = R.Rule(K, score=G, n_groups=4, top_groups=2, group_best=2)
    x, wg, b, g = inputs(T, d, E, F16, 6, 0.02)
    r = make(rule, wg, b, T, backward=True)
    idx, w, lg, count = outs(T - 1, K, E)
    dw, dl = grads(T, K, E, g, True)
    dx, dwg = torch.empty_like(x), torch.empty((E, d), device="cuda")

    def fwd():
        r.route(x, idx, w, lg, count)

    def bwd():
        r.backward(x, lg, idx, dw, dx, dwg, dl)

    def snap():
        torch.cuda.synchronize()
        return [t.clone() for t in (idx, w, lg, count, dx, dwg)]

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        fwd()
        bwd()
    torch.cuda.synchronize()
    graphs = []
    for f in (fwd, bwd):
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            f()
    for i in range(4):
        x.copy_(torch.randn((T, d), generator=g))
        fwd()
        bwd()
        want = snap()
        for t in (idx, w, lg, count, dx, dwg):
            t.fill_(-3)
        graphs[0].replay()
        graphs[1].replay()
        for name, a, b_ in zip(("idx", "w", "logits", "count", "d_x", "d_wg"), snap(), want):
            assert torch.equal(a, b_), (i, name)
    r.destroy()
