"""The layer norm, a routing rule and the layer's experts together, as a model
uses them: serving (norm, a step routed by the router, every path of the
layer) and tuning the gate (forward, a loss on the weights, backward through
routing and norm to the residual stream)."""
import numpy as np
import pytest

from oracle import moe_oracle as O
from oracle import routing_oracle as R
from synth import configs as C

import gpu_support as S
from test_gpu_router import check as check_route, logit_bound, make, outs

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

U = 2.0 ** -24
D, F, E, K = 320, 448, 12, 3
TAGS = (C.TAG_FP16, C.TAG_MISS_INT4, C.TAG_INT4, C.TAG_MISS_INT2) * 3
RULE = R.Rule(K, score=R.SIGMOID, n_groups=4, top_groups=3, group_best=2, scale=2.5)


@pytest.fixture(scope="module", autouse=True)
def _need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2411_01433_amd as P
    P.lib()
    yield


def _workload(T, t1=0.5, t2=0.8):
    return C.Workload(name=f"routed_t{T}", seed=31, d_model=D, d_ff=F, n_experts=E, top_k=K,
                      n_tokens=T, t1=t1, t2=t2, fixed_tags=TAGS)


def _layer(T, rule=RULE, bias=0.05):
    wl = _workload(T)
    w = S.device_layer_weights(wl, 0)
    L = S.make_layer(wl, TAGS, w, max_tokens=max(T, 2))
    b = (torch.randn(E, generator=torch.Generator().manual_seed(2)) * bias).cuda() if bias else None
    return wl, w, L, make(rule, w[0], b, max(T, 2)), b


def _expected(wl, rule, x, wg, b):
    idx, w, l, _ = R.route(rule, x, wg, b)
    share = np.stack([R.shares(rule, l[t], idx[t]) for t in range(len(l))])
    prec = np.stack([R.eq2_precisions(share[t], idx[t], TAGS, wl.t1, wl.t2) for t in range(len(l))])
    # no score lies within the rounding of a threshold
    for t in range(len(l)):
        order = sorted(range(K), key=lambda k: -share[t][k])
        run = np.cumsum([share[t][k] for k in order])
        assert min(np.abs(run - wl.t1).min(), np.abs(run - wl.t2).min()) > 1e-6
    return O.Routing(np.maximum(idx, 0), w, prec, l), idx


def _check(wl, L, r, rule, b, wg, x, call, residual=None):
    T = x.shape[0]
    idx = torch.empty((T, K), dtype=torch.int32, device="cuda")
    w = torch.empty((T, K), device="cuda")
    prec = torch.empty((T, K), dtype=torch.int8, device="cuda")
    y = torch.empty((T, D), device="cuda")
    call(x, y, idx, w, prec)
    torch.cuda.synchronize()
    x16 = x.cpu().numpy()
    want, ref_idx = _expected(wl, rule, x16, wg.cpu().numpy(), None if b is None else b.double().cpu().numpy())
    assert np.array_equal(idx.cpu().numpy(), ref_idx)
    assert np.array_equal(prec.cpu().numpy(), want.prec)
    # the gate values as in the routing tests, the output as in the layer's
    err = logit_bound(x, wg).max() + 64 * U * (1 + np.abs(want.logits).max())
    np.testing.assert_allclose(w.cpu().numpy(), want.w, rtol=2 * err)
    ref = O.layer_output(x16, S.HostExperts(wl, 0, TAGS), want)
    assert S.normwise(y.cpu().numpy(), ref).max() <= S.TOL
    return y, idx, w, prec


@pytest.mark.parametrize("T,entry", [(1, "decode_step"), (4, "decode_step"), (9, "decode_step"),
                                     (64, "decode_step"), (5, "decode_step_noalloc"),
                                     (1, "prefill"), (37, "prefill"), (200, "prefill")])
def test_layer_steps_by_the_router(T, entry):
    wl, w, L, r, b = _layer(T)
    x = torch.from_numpy(C.hidden_states(wl)).cuda()
    y0 = torch.empty((T, D), device="cuda")
    getattr(L, entry)(x, y0)
    L.set_router(r)
    _check(wl, L, r, RULE, b, w[0], x, getattr(L, entry))
    # the layer's own gate again, with its bits
    L.set_router(None)
    y1 = torch.empty_like(y0)
    getattr(L, entry)(x, y1)
    assert torch.equal(y0, y1)
    L.destroy()
    r.destroy()


def test_router_of_the_layers_own_rule_gives_its_routing():
    T = 50
    rule = R.Rule(K)
    wl, w, L, r, _ = _layer(T, rule, bias=0)
    x = torch.from_numpy(C.hidden_states(wl)).cuda()
    a = [torch.empty((T, K), dtype=t, device="cuda") for t in (torch.int32, torch.float32, torch.int8)]
    c = [torch.empty_like(t) for t in a]
    y = torch.empty((T, D), device="cuda")
    L.prefill(x, y, *a)
    L.set_router(r)
    y2 = torch.empty_like(y)
    L.prefill(x, y2, *c)
    assert torch.equal(a[0], c[0]) and torch.equal(a[2], c[2])
    assert (a[1] - c[1]).abs().max().item() <= 1e-5
    assert S.normwise(y2.cpu().numpy(), y.cpu().numpy()).max() <= S.TOL
    L.destroy()
    r.destroy()


def test_tokens_without_experts():
    """Masked down to two experts: the third slot is empty; with none left the
    layer gives zeros."""
    for T, entry in ((1, "decode_step"), (8, "decode_step"), (64, "decode_step"), (70, "prefill")):
        wl, w, L, r, b = _layer(T)
        x = torch.from_numpy(C.hidden_states(wl)).cuda()
        L.set_router(r)
        b.fill_(-float("inf"))
        b[4], b[10] = 0.0, 0.1
        _, idx, gw, prec = _check(wl, L, r, RULE, b, w[0], x, getattr(L, entry))
        assert (idx[:, 2] == -1).all() and (gw[:, 2] == 0).all() and (prec[:, 2] == 2).all()
        b.fill_(-float("inf"))
        y = torch.full((T, D), 9.0, device="cuda")
        getattr(L, entry)(x, y)
        assert (y == 0).all()
        L.destroy()
        r.destroy()


@pytest.mark.parametrize("T", [2, 20, 90])
def test_norm_and_routed_layers_on_the_residual_stream(T):
    """Two layers: x = layer norm(h), h += layer(x) by the residual entry point
    (its RMS-normed x_next is not used), each layer routed by a router; against
    the oracles, teacher-forced on the library's own x and h."""
    import paper_2411_01433_amd as P
    wl, w, L, r, b = _layer(T)
    L.set_router(r)
    g = torch.Generator().manual_seed(3)
    h = torch.randn((T, D), generator=g).cuda()
    gain, bias = (1 + 0.1 * torch.randn(D, generator=g)).cuda(), (0.1 * torch.randn(D, generator=g)).cuda()
    x, xn = (torch.empty((T, D), dtype=torch.float16, device="cuda") for _ in range(2))
    for _ in range(2):
        before = h.clone()
        P.layernorm(h, x, gain, bias)
        ref = R.layernorm(*(t.double().cpu().numpy() for t in (h, gain, bias)))
        assert np.abs(x.double().cpu().numpy() - ref).max() <= (2.0 ** -11 + 64 * U) * np.abs(ref).max()
        (L.prefill_residual if T > 64 else L.decode_step_residual)(x, h, xn)
        torch.cuda.synchronize()
        want, _ = _expected(wl, RULE, x.cpu().numpy(), w[0].cpu().numpy(), b.double().cpu().numpy())
        y = O.layer_output(x.cpu().numpy(), S.HostExperts(wl, 0, TAGS), want)
        assert S.normwise((h - before).cpu().numpy(), y).max() <= S.TOL
        if T <= 64:  # the pre-norm entry point of a routed layer: norm, then the step
            h2, x2 = before.clone(), torch.empty_like(x)
            L.decode_step_prenorm(h2, x2)
            x3, h3 = torch.empty_like(x), before.clone()
            P.rmsnorm(before, x3)
            L.decode_step_residual(x3, h3, xn)
            assert torch.equal(x2, x3) and torch.equal(h2, h3)
    L.destroy()
    r.destroy()


def test_captured_routed_step():
    T = 9
    wl, w, L, r, b = _layer(T)
    L.set_router(r)
    x = torch.from_numpy(C.hidden_states(wl)).cuda()
    y = torch.empty((T, D), device="cuda")
    L.decode_step(x, y)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        L.decode_step(x, y)
    for i in range(3):
        x.copy_(torch.from_numpy(C.hidden_states(wl, stream=i + 1)))
        L.decode_step(x, y)
        torch.cuda.synchronize()
        want = y.clone()
        y.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, want), i
    L.destroy()
    r.destroy()


def test_set_router_refusals():
    import paper_2411_01433_amd as P
    wl, w, L, r, b = _layer(8)
    wg = w[0]
    cases = [
        P.MoeRouter(D, E, K, 8, wg.bfloat16(), dtype=torch.bfloat16),
        P.MoeRouter(D, E, K - 1, 8, wg),
        P.MoeRouter(D, E - 1, K, 8, wg[:-1].contiguous()),
        P.MoeRouter(256, E, K, 8, wg[:, :256].contiguous()),
        P.MoeRouter(D, E, K, 7, wg),
    ]
    for c in cases:
        with pytest.raises(P.MoeError):
            L.set_router(c)
        c.destroy()
    L.set_router(r)
    with pytest.raises(P.MoeError, match="still route"):
        r.destroy()
    L.set_router(r)          # again: still one use
    L.destroy()
    r.destroy()              # the layer's end let go of it


def test_tuning_a_gate_by_the_experts_loads():
    """Norm, routing, a loss on weights and logits, and its gradients back to
    the residual stream, the gate and the norm's gain, against 64 bits."""
    import paper_2411_01433_amd as P
    T = 150
    g = torch.Generator().manual_seed(9)
    h = torch.randn((T, D), generator=g).cuda()
    gain, bias = (1 + 0.1 * torch.randn(D, generator=g)).cuda(), (0.1 * torch.randn(D, generator=g)).cuda()
    wg = (torch.randn((E, D), generator=g) * 0.05).half().cuda()
    b = torch.zeros(E, device="cuda")
    r = make(RULE, wg, b, T, backward=True)
    x = torch.empty((T, D), dtype=torch.float16, device="cuda")
    idx, w, lg, count = outs(T - 1, K, E)
    up = torch.randn((T, K), generator=g).cuda()
    P.layernorm(h, x, gain, bias)
    spread = []
    for _ in range(8):  # the bias evens the loads out: loads of the last call steer the next
        r.route(x, idx, w, lg, count)
        c = count.float()
        assert int(c.sum()) == T * K
        spread.append((c.max() - c.min()).item())
        b.add_(0.01 * torch.sign(c.mean() - c))
    check_route(RULE, x, wg, b, r)
    r.route(x, idx, w, lg, count)
    dx, dwg = torch.empty_like(x), torch.empty((E, D), device="cuda")
    dh, dg, db = torch.ones_like(h), torch.empty_like(gain), torch.empty_like(bias)
    r.backward(x, lg, idx, up, dx, dwg, lg * 0.001)
    P.layernorm_backward(dx, h, dh, gain, dg, db, accumulate=True)
    torch.cuda.synchronize()
    n = lambda t: t.double().cpu().numpy()
    rx, rw, _ = R.route_backward(RULE, n(x), n(wg), n(lg), idx.cpu().numpy(), n(up), n(lg) * 0.001)
    rh, rg, rb = R.layernorm_backward(rx, n(h), n(gain))
    # d_x is rounded to fp16 in between: half a step of it in every sum
    for got, ref, name in ((n(dx), rx, "x"), (n(dh) - 1.0, rh, "h"), (n(dg), rg, "gain"), (n(db), rb, "bias")):
        off = np.linalg.norm(got - ref) / np.linalg.norm(ref)
        assert off <= 2.0 ** -11, (name, off)
    assert np.linalg.norm(n(dwg) - rw) / np.linalg.norm(rw) <= 1e-5
    r.destroy()


def test_a_destroyed_router_is_not_taken():
    """... for the layer's own gate: the layer refuses it and keeps its router."""
    wl, w, L, r, b = _layer(4)
    L.set_router(r)
    other = make(RULE, w[0], b, 4)
    other.destroy()
    with pytest.raises(ValueError, match="destroyed"):
        L.set_router(other)
    with pytest.raises(Exception, match="still route"):
        r.destroy()
    L.set_router(None)
    r.destroy()
    L.destroy()
