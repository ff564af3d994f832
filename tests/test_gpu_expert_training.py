"""The operators as a tuning step uses them: layer norm, routing, rows sorted by
expert, the experts' products with a SwiGLU between them, the weighted sum;
then every gradient back to the residual stream, and the clipping.  Against the
same in 64 bits, whose selection is the library's.

Bounds.  The step rounds to fp16 between its products, half a step (2^-11) each
time, along a chain of at most 12 roundings forward and back; they add up as
independent errors of whole tensors do, so 12 * 2^-11 of a gradient's norm holds
them with room."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

TOL = 12 * 2.0 ** -11


@pytest.fixture(scope="module", autouse=True)
def _need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2411_01433_amd as P
    P.lib()
    yield


def _near(got, ref):
    err = (got.double() - ref).norm() / ref.norm()
    assert err <= TOL, float(err)


def _silu_grad(a):
    s = torch.sigmoid(a)
    return s * (1 + a * (1 - s))


@pytest.mark.parametrize("T,d,f,E,K", [(1, 64, 128, 4, 2), (50, 128, 192, 8, 2), (300, 256, 320, 6, 3)])
def test_tuning_step(T, d, f, E, K):
    import paper_2411_01433_amd as P
    g = torch.Generator().manual_seed(T)
    rand = lambda *s, std=1.0: std * torch.randn(s, generator=g)
    h = rand(T, d).cuda()
    gain, bias = (1 + rand(d, std=0.1)).cuda(), rand(d, std=0.1).cuda()
    wg = rand(E, d, std=0.05).half().cuda()
    w1, w3 = (rand(E, f, d, std=d ** -0.5).half().cuda() for _ in range(2))
    w2 = rand(E, d, f, std=f ** -0.5).half().cuda()
    dout = rand(T, d, std=0.1).cuda()

    # forward
    f16 = lambda *s: torch.empty(s, dtype=torch.float16, device="cuda")
    x = f16(T, d)
    P.layernorm(h, x, gain, bias)
    router = P.MoeRouter(d, E, K, T, wg, backward=True)
    idx = torch.empty((T, K), dtype=torch.int32, device="cuda")
    wt, logits = torch.empty((T, K), device="cuda"), torch.empty((T, E), device="cuda")
    count = torch.empty(E, dtype=torch.int32, device="cuda")
    router.route(x, idx, wt, logits, count)
    order = torch.argsort(idx.view(-1), stable=True)
    token, R = order // K, T * K
    xs = x[token]
    a, b, o = f16(R, f), f16(R, f), f16(R, d)
    P.grouped_product(xs, w1, a, count)
    P.grouped_product(xs, w3, b, count)
    hid = (torch.nn.functional.silu(a.float()) * b.float()).half()
    P.grouped_product(hid, w2, o, count)
    ws = wt.view(-1)[order]
    y = torch.zeros((T, d), device="cuda").index_add_(0, token, ws[:, None] * o.float())

    # backward
    do = (ws[:, None] * dout[token]).half()
    dws = (dout[token] * o.float()).sum(-1)
    dhid, dxs1, dxs3 = f16(R, f), f16(R, d), f16(R, d)
    dw1, dw3, dw2 = (torch.empty(w.shape, device="cuda") for w in (w1, w3, w2))
    P.grouped_product_backward(do, hid, w2, count, dhid, dw2)
    da = (dhid.float() * b.float() * _silu_grad(a.float())).half()
    db = (dhid.float() * torch.nn.functional.silu(a.float())).half()
    P.grouped_product_backward(da, xs, w1, count, dxs1, dw1)
    P.grouped_product_backward(db, xs, w3, count, dxs3, dw3)
    dx = torch.zeros((T, d), device="cuda").index_add_(0, token, dxs1.float() + dxs3.float())
    dwt = torch.empty(R, device="cuda")
    dwt[order] = dws
    dxr, dwg = f16(T, d), torch.empty((E, d), device="cuda")
    router.backward(x, logits, idx, dwt.view(T, K), dxr, dwg)
    dh, dgain, dbias = torch.empty_like(h), torch.empty(d, device="cuda"), torch.empty(d, device="cuda")
    P.layernorm_backward((dx + dxr.float()).half(), h, dh, gain, dgain, dbias)
    grads = [dw1, dw3, dw2, dwg, dgain, dbias]
    raw = [t.clone() for t in grads]
    norm = torch.empty(1, device="cuda")
    P.MoeGradients(grads).clip(0.5, norm)

    # the same in 64 bits, on the CPU
    par = [t.double().cpu().requires_grad_() for t in (h, gain, bias, wg, w1, w3, w2)]
    h6, gain6, bias6, wg6, w16, w36, w26 = par
    x6 = torch.nn.functional.layer_norm(h6, (d,), gain6, bias6, 1e-5)
    p = torch.softmax(x6 @ wg6.T, -1).gather(1, idx.long().cpu())
    p = p / p.sum(-1, keepdim=True)
    y6 = 0
    for k in range(K):
        e = idx[:, k].long().cpu()
        a6 = torch.bmm(w16[e], x6[:, :, None])[..., 0]
        b6 = torch.bmm(w36[e], x6[:, :, None])[..., 0]
        hid6 = torch.nn.functional.silu(a6) * b6
        y6 = y6 + p[:, k, None] * torch.bmm(w26[e], hid6[:, :, None])[..., 0]
    (y6 * dout.double().cpu()).sum().backward()
    _near(y.cpu(), y6.detach())
    _near(dh.cpu(), h6.grad)
    for got, t in zip(raw, (w16, w36, w26, wg6, gain6, bias6)):
        _near(got.cpu(), t.grad)
    total = torch.sqrt(sum(t.double().square().sum() for t in raw))
    assert abs(norm.item() - total.item()) <= 2e-7 * total.item()
    c = min(1.0, 0.5 / (total.item() + 1e-6))
    for got, t in zip(grads, raw):
        assert torch.allclose(got.double(), c * t.double(), rtol=1e-6, atol=0)
    router.destroy()


def test_serving_in_four_bits():
    """A router's tokens through experts quantised once, at 16-bit and at 4-bit
    activations, against the values that the quantiser returned."""
    import paper_2411_01433_amd as P
    T, d, f, E, K = 70, 192, 256, 8, 2
    g = torch.Generator().manual_seed(2)
    x = torch.randn((T, d), generator=g).half().cuda()
    wg = (0.1 * torch.randn((E, d), generator=g)).half().cuda()
    w = (d ** -0.5 * torch.randn((E, f, d), generator=g)).half().cuda()
    idx = torch.empty((T, K), dtype=torch.int32, device="cuda")
    wt, count = torch.empty((T, K), device="cuda"), torch.empty(E, dtype=torch.int32, device="cuda")
    router = P.MoeRouter(d, E, K, T, wg)
    router.route(x, idx, wt, None, count)
    order = torch.argsort(idx.view(-1), stable=True)
    xs = x[order // K]
    wv = torch.empty_like(w)
    u8 = lambda *s: torch.empty(s, dtype=torch.uint8, device="cuda")
    wc, ws = u8(E, f, d // 2), u8(E, f, d // 32)
    P.mx_quantize(w.view(-1, d), wc.view(-1, d // 2), ws.view(-1, d // 32), wv.view(-1, d))
    xc, xsc, xv = u8(T * K, d // 2), u8(T * K, d // 32), torch.empty_like(xs)
    P.mx_quantize(xs, xc, xsc, xv)
    e = idx.view(-1)[order].long().cpu()
    y = torch.empty((T * K, f), dtype=torch.float16, device="cuda")
    for acts, xin, scales in ((xs, xs, None), (xv, xc, xsc)):
        P.mx_product(xin, wc, ws, y, count, scales)
        ref = torch.bmm(wv.double().cpu()[e], acts.double().cpu()[:, :, None])[..., 0]
        _near(y.cpu(), ref)
    # and 4-bit weights are what they are called: within half a step of the grid
    assert ((wv.double() - w.double()).norm() / w.double().norm()).item() < 0.2
    router.destroy()
