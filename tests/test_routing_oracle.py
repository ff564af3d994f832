"""Pins of the routing and layer norm oracle: worked values, and gradients
against central differences of the forward functions."""
import numpy as np
import pytest

from oracle import routing_oracle as R


def test_worked_softmax_and_sigmoid():
    l = np.log(np.array([1.0, 4.0, 2.0, 3.0]))
    idx = R.select(R.Rule(2), l)
    assert idx.tolist() == [1, 3]
    np.testing.assert_allclose(R.weights(R.Rule(2), l, idx), [4 / 7, 3 / 7], rtol=1e-14)
    np.testing.assert_allclose(R.weights(R.Rule(2, renormalize=False), l, idx), [0.4, 0.3], rtol=1e-14)
    r = R.Rule(2, score=R.SIGMOID, renormalize=False, scale=2.0)
    np.testing.assert_allclose(R.weights(r, l, idx), [2 * 4 / 5, 2 * 3 / 4], rtol=1e-14)


def test_bias_moves_the_selection_and_not_the_weight():
    l = np.array([0.0, 1.0, 2.0, 3.0])
    r = R.Rule(2, score=R.SIGMOID, renormalize=False)
    idx = R.select(r, l, np.array([1.0, 0.0, 0.0, 0.0]))
    assert idx.tolist() == [0, 3]
    np.testing.assert_allclose(R.weights(r, l, idx), [0.5, 1 / (1 + np.exp(-3.0))], rtol=1e-14)


def test_groups_by_one_and_by_two():
    l = np.array([3.0, -9.0, 2.0, 2.0, 0.0, 0.0])
    one = R.Rule(1, score=R.SIGMOID, n_groups=3, top_groups=1, group_best=1)
    two = R.Rule(1, score=R.SIGMOID, n_groups=3, top_groups=1, group_best=2)
    assert R.select(one, l).tolist() == [0]
    assert R.select(two, l).tolist() == [2]  # 0.88 + 0.88 beat 0.95 + 0.0001; the tie to the lower


def test_masked_and_missing_experts():
    l = np.array([1.0, np.nan, 5.0, np.inf])
    r = R.Rule(3)
    assert R.select(r, l, np.array([0.0, 0.0, -np.inf, 0.0])).tolist() == [0, -1, -1]
    assert R.weights(r, l, np.array([0, -1, -1])).tolist() == [1.0, 0.0, 0.0]
    assert R.select(r, np.full(4, np.nan)).tolist() == [-1, -1, -1]


def test_ranks_of_the_precision_rule():
    # slots by key; shares not in that order
    prec = R.eq2_precisions([0.2, 0.5, 0.3], np.array([0, 1, 2]), [3, 3, 3], 0.6, 0.7)
    assert prec.tolist() == [2, 0, 0]
    assert R.eq2_precisions([1.0, 0.0], np.array([1, -1]), [3, 3], 0.5, 1.0).tolist() == [0, 2]


RULES = [R.Rule(3), R.Rule(3, renormalize=False, scale=2.5), R.Rule(3, score=R.SIGMOID, scale=2.5),
         R.Rule(2, score=R.SIGMOID, renormalize=False)]


@pytest.mark.parametrize("rule", RULES, ids=["softmax", "softmax_all", "sigmoid", "sigmoid_raw"])
def test_route_gradients_by_differences(rule):
    rng = np.random.default_rng(7)
    T, d, E = 3, 6, 5
    x, wg = rng.normal(size=(T, d)), rng.normal(size=(E, d))
    dw, dl = rng.normal(size=(T, rule.top_k)), rng.normal(size=(T, E))
    idx, _, l, _ = R.route(rule, x, wg)

    def loss(x, wg):
        l = x @ wg.T
        return sum((R.weights(rule, l[t], idx[t]) * dw[t]).sum() for t in range(T)) + (l * dl).sum()

    dx, dwg, _ = R.route_backward(rule, x, wg, l, idx, dw, dl)
    h = 1e-5
    for a, g, f in ((x, dx, lambda v: loss(v, wg)), (wg, dwg, lambda v: loss(x, v))):
        for i in np.ndindex(a.shape):
            up, dn = a.copy(), a.copy()
            up[i] += h
            dn[i] -= h
            assert abs((f(up) - f(dn)) / (2 * h) - g[i]) < 1e-8


@pytest.mark.parametrize("affine", [True, False])
def test_layernorm_gradients_by_differences(affine):
    rng = np.random.default_rng(8)
    T, d = 3, 7
    h, up = rng.normal(size=(T, d)), rng.normal(size=(T, d))
    gain = rng.normal(size=d) if affine else None
    bias = rng.normal(size=d) if affine else None
    dh, dg, db = R.layernorm_backward(up, h, gain)
    eps = 1e-5

    def diff(f, a, i):
        hi, lo = a.copy(), a.copy()
        hi[i] += eps
        lo[i] -= eps
        return (f(hi) - f(lo)) / (2 * eps)

    for i in np.ndindex(h.shape):
        assert abs(diff(lambda v: (R.layernorm(v, gain, bias) * up).sum(), h, i) - dh[i]) < 1e-7
    if affine:
        for i in range(d):
            assert abs(diff(lambda v: (R.layernorm(h, v, bias) * up).sum(), gain, i) - dg[i]) < 1e-7
            assert abs(diff(lambda v: (R.layernorm(h, gain, v) * up).sum(), bias, i) - db[i]) < 1e-7
