"""Refusals of the grouped products, the MXFP4 entry points and the gradient
lists (runs without a GPU): every bad argument is an error before any work is
enqueued.  And the oracle's own pins."""
import ctypes

import numpy as np
import pytest

from oracle import experts_oracle as X
from paper_2411_01433_amd import binding as B

P16, P8, P2, P1 = (ctypes.c_void_p(0x1000 + k) for k in (0, 8, 2, 1))
SIZES = dict(type=B.MOE_F16, n_rows=4, d_in=64, d_out=128, n_experts=2)


def _sizes(**kw):
    return [ctypes.c_int32(v) for v in {**SIZES, **kw}.values()]


BAD_SIZES = [
    dict(type=2), dict(type=-1), dict(n_rows=-1), dict(n_rows=(1 << 21) + 1), dict(d_in=0),
    dict(d_in=96), dict(d_in=-64), dict(d_in=65600), dict(d_out=0), dict(d_out=100),
    dict(d_out=65600), dict(n_experts=0), dict(n_experts=513),
]


def _product(x=P16, w=P16, count=P16, y=P16, **kw):
    return B.lib().moe_grouped_product(x, w, count, y, *_sizes(**kw), None)


def _backward(dy=P16, x=P16, w=P16, count=P16, dx=P16, dw=P16, **kw):
    return B.lib().moe_grouped_product_backward(dy, x, w, count, dx, dw, 0, *_sizes(**kw), None)


def _mx(x=P16, xs=None, w=P16, ws=P16, count=P16, y=P16, **kw):
    return B.lib().moe_mx_product(x, xs, w, ws, count, y, *_sizes(**kw), None)


@pytest.mark.parametrize("call", [_product, _backward, _mx])
@pytest.mark.parametrize("bad", BAD_SIZES)
def test_sizes(call, bad):
    assert call(**bad) == B.MOE_EINVAL and B.lib().moe_last_error()


@pytest.mark.parametrize("call", [_product, _backward, _mx])
def test_counts(call):
    assert call(count=None) == B.MOE_EINVAL  # two experts
    assert call(count=P2) == B.MOE_EINVAL


def test_product_pointers():
    for name in ("x", "w", "y"):
        assert _product(**{name: None}) == B.MOE_EINVAL
        assert _product(**{name: P8}) == B.MOE_EINVAL
    assert _product(n_rows=0, w=None) == B.MOE_EINVAL
    # no rows: no work, so nothing touches the device
    assert _product(n_rows=0, x=None, y=None) == B.MOE_OK


def test_backward_pointers():
    for name in ("dy", "x", "w"):
        assert _backward(**{name: None}) == B.MOE_EINVAL
    for name in ("dy", "x", "w", "dx", "dw"):
        assert _backward(**{name: P8}) == B.MOE_EINVAL
    assert _backward(dx=None, dw=None) == B.MOE_EINVAL
    assert _backward(n_rows=0, dy=None, x=None, dw=None) == B.MOE_OK
    assert B.lib().moe_grouped_product_backward(None, None, None, P16, None, P16, 1,
                                                *_sizes(n_rows=0), None) == B.MOE_OK


def test_mx_product_pointers():
    for name in ("x", "w", "ws", "y"):
        assert _mx(**{name: None}) == B.MOE_EINVAL
    for name in ("x", "w", "y"):
        assert _mx(**{name: P8}) == B.MOE_EINVAL
    for odd in (P1, P2):
        assert _mx(ws=odd) == B.MOE_EINVAL
        assert _mx(xs=odd) == B.MOE_EINVAL
    assert _mx(n_rows=0, x=None, y=None) == B.MOE_OK


@pytest.mark.parametrize("bad", [
    dict(type=2), dict(rows=-1), dict(rows=1 << 31), dict(rows=1 << 30), dict(cols=0),
    dict(cols=32), dict(cols=96), dict(cols=65600), dict(v=None), dict(codes=None),
    dict(scales=None), dict(v=P8), dict(codes=P8), dict(scales=P1), dict(values=P8),
])
def test_mx_quantize(bad):
    a = {**dict(v=P16, type=0, rows=2, cols=64, codes=P16, scales=P16, values=None), **bad}
    assert B.lib().moe_mx_quantize(a["v"], a["type"], a["rows"], a["cols"], a["codes"],
                                   a["scales"], a["values"], None) == B.MOE_EINVAL


def test_mx_quantize_of_no_rows():
    assert B.lib().moe_mx_quantize(None, 0, 0, 64, None, None, None, None) == B.MOE_OK


def _init(grads=(0x1000, 0x2000), outs=None, sizes=(64, 64), types=(2, 2), n=None):
    k = len(grads)
    out = ctypes.c_void_p(123)
    st = B.lib().moe_gradients_init(
        k if n is None else n, (ctypes.c_void_p * k)(*grads),
        None if outs is None else (ctypes.c_void_p * k)(*outs), (ctypes.c_int64 * k)(*sizes),
        (ctypes.c_int32 * k)(*types), None, ctypes.byref(out))
    assert out.value is None
    return st


@pytest.mark.parametrize("bad", [
    dict(n=0), dict(n=-1), dict(n=65537), dict(types=(2, 3)), dict(types=(-1, 2)),
    dict(sizes=(64, -1)), dict(sizes=(64, 1 << 38)), dict(sizes=(1 << 37, 1 << 37)),
    dict(grads=(0x1000, None)), dict(outs=(0x3000, None)), dict(grads=(0x1000, 0x2002)),
    dict(types=(2, 0), grads=(0x1000, 0x2001)), dict(outs=(0x3000, 0x4002)),
    dict(grads=(0x1000, 0x1000)),               # the same tensor twice
    dict(grads=(0x1000, 0x10fc)),               # one element shared
    dict(outs=(0x2000, 0x3000)),                # an output over another's input
    dict(outs=(0x1004, 0x3000)),                # over its own, shifted
    dict(outs=(0x3000, 0x3000)),
])
def test_gradients_init(bad):
    assert _init(**bad) == B.MOE_EINVAL and B.lib().moe_last_error()


def test_gradients_handles():
    L, bogus = B.lib(), ctypes.c_void_p(0xdead0)
    z = (ctypes.c_int64 * 1)(4)
    t = (ctypes.c_int32 * 1)(2)
    g = (ctypes.c_void_p * 1)(0x1000)
    out = ctypes.c_void_p()
    assert L.moe_gradients_init(1, g, None, z, t, None, None) == B.MOE_EINVAL
    assert L.moe_gradients_init(1, None, None, z, t, None, ctypes.byref(out)) == B.MOE_EINVAL
    assert L.moe_gradients_init(1, g, None, None, t, None, ctypes.byref(out)) == B.MOE_EINVAL
    assert L.moe_gradients_init(1, g, None, z, None, None, ctypes.byref(out)) == B.MOE_EINVAL
    for h in (None, bogus):
        assert L.moe_gradients_norm(h, P16, None) == B.MOE_ESTATE
        assert L.moe_gradients_scale(h, 1.0, P16, None) == B.MOE_ESTATE
        assert L.moe_gradients_clip(h, 1.0, P16, None) == B.MOE_ESTATE
    assert L.moe_gradients_destroy(bogus) == B.MOE_ESTATE
    assert L.moe_gradients_destroy(None) == B.MOE_EINVAL


# ---- the oracle ---------------------------------------------------------------

def test_oracle_mx_worked_example():
    """Largest 7 -> e = 0: 7 saturates to 6; ties 0.25 -> 0, 0.75 -> 1, 1.25 -> 1,
    1.75 -> 2, 2.5 -> 2, 3.5 -> 4, 5 -> 4."""
    v = np.zeros((1, 64))
    v[0, :9] = [7, 0.25, 0.75, -1.25, 1.75, 2.5, -3.5, 5, 0.26]
    v[0, 32] = -0.75  # second block: e = -3
    codes, scales = X.mx_quantize(v)
    assert scales.tolist() == [[127, 124]]
    got = X.mx_values(codes, scales)[0]
    assert got[:9].tolist() == [6, 0, 1, -1, 2, 2, -4, 4, 0.5]
    assert got[32] == -0.75 and not got[9:32].any() and not got[33:].any()
    assert codes[0, 0] == 0x07 and codes[0, 1] == 0xA2 and codes[0, 16] == 0x0F


def test_oracle_mx_zero_and_least_scale():
    v = np.zeros((2, 64))
    v[1, 0] = 2.0 ** -133
    codes, scales = X.mx_quantize(v)
    assert scales.tolist() == [[0, 0], [0, 0]] and not codes[0].any()
    assert X.mx_values(codes, scales)[1, 0] == 0  # 2^-6 of the least scale
    v[1, 0] = 2.0 ** -127
    assert X.mx_values(*X.mx_quantize(v))[1, 0] == 2.0 ** -127


def test_oracle_products_against_differences():
    """d_x and d_w are the derivatives of sum(dy * y)."""
    rng = np.random.default_rng(1)
    x, w = rng.standard_normal((6, 4)), rng.standard_normal((3, 5, 4))
    counts, dy = [2, 0, 3], rng.standard_normal((6, 5))
    f = lambda x, w: (dy * X.grouped_product(x, w, counts, np.zeros((6, 5)))[0]).sum()
    dx, dw, _, _ = X.grouped_product_backward(dy, x, w, counts, np.zeros_like(x), np.zeros_like(w))
    for a, da in ((x, dx), (w, dw)):
        for i in np.ndindex(a.shape):
            old, h = a[i], 1e-6
            a[i] = old + h
            up = f(x, w)
            a[i] = old - h
            down = f(x, w)
            a[i] = old
            assert abs((up - down) / (2 * h) - da[i]) < 1e-8
    assert not dx[5].any() and not dw[1].any()


def test_oracle_clip():
    n, out = X.clip([np.array([3.0]), np.array([4.0])], 1.0)
    assert n == 5 and abs(out[1][0] - 0.8) < 1e-6
    assert X.clip([np.array([3.0])], 10.0)[1][0][0] == 3.0
    assert X.clip([np.array([np.inf, 2.0])], 1.0)[1][0][1] == 2.0
