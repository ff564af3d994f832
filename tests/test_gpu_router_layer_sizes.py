"""Layers routed by a router at the sizes of every selection kernel: more than
16 experts (a kernel for the logits, one for the selection), more than 2048
tokens (open tokens on a list), a softmax beside a bias (blocks of waves for a
token), against the oracles."""
import numpy as np
import pytest

from oracle import moe_oracle as O
from oracle import routing_oracle as R
from synth import configs as C

import gpu_support as S
from test_gpu_router import U, logit_bound, make

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

D, F = 128, 64


@pytest.fixture(scope="module", autouse=True)
def _need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2411_01433_amd as P
    P.lib()
    yield


CASES = [
    # T, E, entry, bias, masked experts, rule
    (1, 60, "decode_step", 0.02, 0, R.Rule(4, score=R.SIGMOID, n_groups=6, top_groups=3, group_best=2)),
    (8, 17, "decode_step_noalloc", 0, 0, R.Rule(8, renormalize=False, scale=2.5)),
    (33, 64, "decode_step", 0.002, 0, R.Rule(8)),
    (64, 60, "decode_step", 0.02, 57, R.Rule(4, score=R.SIGMOID, scale=2.5)),
    (300, 40, "prefill", 0.02, 0, R.Rule(5, score=R.SIGMOID, n_groups=5, top_groups=2, group_best=2)),
    (600, 60, "prefill", 0.002, 0, R.Rule(4, renormalize=False)),
    (2100, 64, "prefill", 0.02, 0, R.Rule(8, score=R.SIGMOID, n_groups=8, top_groups=4, group_best=2)),
    (2300, 60, "prefill", 0.02, 58, R.Rule(4, score=R.SIGMOID)),
    (4100, 24, "prefill", 0, 0, R.Rule(2)),
]


@pytest.mark.parametrize("T,E,entry,bias,masked,rule", CASES, ids=[f"t{c[0]}_e{c[1]}" for c in CASES])
def test_routed_layer(T, E, entry, bias, masked, rule):
    K = rule.top_k
    tags = ((C.TAG_FP16, C.TAG_MISS_INT4, C.TAG_INT4, C.TAG_MISS_INT2) * 16)[:E]
    wl = C.Workload(name=f"routed_t{T}_e{E}", seed=37, d_model=D, d_ff=F, n_experts=E, top_k=K,
                    n_tokens=T, t1=0.3, t2=0.6, fixed_tags=tags)
    w = S.device_layer_weights(wl, 0)
    L = S.make_layer(wl, tags, w, max_tokens=T)
    g = torch.Generator().manual_seed(T)
    b = (torch.randn(E, generator=g) * bias).cuda() if bias else None
    if masked:
        b[torch.randperm(E, generator=g)[:masked].cuda()] = -float("inf")
    r = make(rule, w[0], b, T)
    L.set_router(r)
    x = torch.from_numpy(C.hidden_states(wl)).cuda()
    idx = torch.full((T + 1, K), -7, dtype=torch.int32, device="cuda")
    gw, prec = torch.full((T + 1, K), -7.0, device="cuda"), torch.full((T + 1, K), -7, dtype=torch.int8, device="cuda")
    y = torch.full((T + 1, D), -7.0, device="cuda")
    getattr(L, entry)(x, y[:T], idx[:T], gw[:T], prec[:T])
    torch.cuda.synchronize()
    for t in (idx, gw, prec, y):
        assert (t[T] == -7).all()
    idx, gw, prec, y = (t[:T].cpu().numpy() for t in (idx, gw, prec, y))
    x64 = x.double().cpu().numpy()
    ref_idx, ref_w, l, _ = R.route(rule, x64, w[0].double().cpu().numpy(),
                                   None if b is None else b.double().cpu().numpy())
    assert np.array_equal(idx, ref_idx)
    # (a slot without an expert: -1, weight 0, skipped)
    assert not masked or ((idx < 0).any() and (prec[idx < 0] == 2).all() and (gw[idx < 0] == 0).all())
    err = logit_bound(x, w[0]).max() + 64 * U * (1 + np.abs(l).max())
    np.testing.assert_allclose(gw, ref_w, rtol=2 * err)
    share = np.stack([R.shares(rule, l[t], idx[t]) for t in range(T)])
    want = np.stack([R.eq2_precisions(share[t], idx[t], tags, wl.t1, wl.t2) for t in range(T)])
    run = np.cumsum(-np.sort(-share, axis=1), axis=1)
    sure = np.minimum(np.abs(run - wl.t1), np.abs(run - wl.t2)).min(1) > 2 * err
    # (two equal shares are ranked by their slots, which rounding may separate)
    gap = -np.diff(-np.sort(-share, axis=1), axis=1)
    sure &= np.where(gap == 0, np.inf, gap).min(1, initial=np.inf) > 2 * err
    assert 2 * sure.sum() > T
    assert np.array_equal(prec[sure], want[sure])
    few = np.unique(np.concatenate([np.arange(min(T, 40)), np.arange(max(0, T - 40), T)]))
    routing = O.Routing(np.maximum(idx, 0)[few], ref_w[few], prec[few], l[few])
    ref = O.layer_output(x.cpu().numpy()[few], S.HostExperts(wl, 0, tags), routing)
    assert S.normwise(y[few], ref).max() <= S.TOL
    # the same bits again
    y2 = torch.empty((T, D), device="cuda")
    getattr(L, entry)(x, y2)
    assert np.array_equal(y2.cpu().numpy(), y)
    L.destroy()
    r.destroy()
