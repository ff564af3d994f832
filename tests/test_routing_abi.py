"""Refusals of the routing and layer norm entry points (runs without a GPU):
every bad argument is an error before any work is enqueued."""
import ctypes

import pytest

from paper_2411_01433_amd import binding as B

P16, ODD = ctypes.c_void_p(0x1000), ctypes.c_void_p(0x1004)


def _desc(**kw):
    d = dict(d_model=256, n_experts=8, top_k=2, max_tokens=4, type=B.MOE_F16,
             score=B.SCORE_SIGMOID, n_groups=4, top_groups=2, group_best=2, renormalize=1,
             scale=2.5, flags=0)
    d.update(kw)
    return B.RouterDesc(**d)


def test_desc_layout_matches_header():
    assert ctypes.sizeof(B.RouterDesc) == 48  # 10 int32, a float, a uint32, no padding


@pytest.mark.parametrize("bad", [
    dict(d_model=0), dict(d_model=100), dict(d_model=16448), dict(n_experts=0),
    dict(n_experts=513, n_groups=1, top_groups=1), dict(top_k=0), dict(top_k=17, n_experts=64),
    dict(top_k=5), dict(top_k=3, top_groups=1), dict(n_groups=0), dict(n_groups=3),
    dict(n_groups=128, n_experts=256), dict(top_groups=0), dict(top_groups=5),
    dict(group_best=0), dict(group_best=3), dict(max_tokens=0), dict(max_tokens=65537),
    dict(type=2), dict(type=-1), dict(score=2), dict(renormalize=2), dict(scale=0.0),
    dict(scale=-1.0), dict(scale=float("nan")), dict(scale=float("inf")), dict(flags=2),
])
def test_router_init_rejects_bad_desc(bad):
    out = ctypes.c_void_p(123)
    desc = _desc(**bad)
    assert B.lib().moe_router_init(ctypes.byref(desc), P16, None, ctypes.byref(out)) == B.MOE_EINVAL
    assert out.value is None and B.lib().moe_last_error()


def test_router_init_rejects_bad_pointers():
    L, out, desc = B.lib(), ctypes.c_void_p(123), _desc()
    assert L.moe_router_init(None, P16, None, ctypes.byref(out)) == B.MOE_EINVAL
    assert L.moe_router_init(ctypes.byref(desc), None, None, ctypes.byref(out)) == B.MOE_EINVAL
    assert L.moe_router_init(ctypes.byref(desc), ODD, None, ctypes.byref(out)) == B.MOE_EINVAL
    assert L.moe_router_init(ctypes.byref(desc), P16, ctypes.c_void_p(0x1002),
                             ctypes.byref(out)) == B.MOE_EINVAL
    assert L.moe_router_init(ctypes.byref(desc), P16, None, None) == B.MOE_EINVAL
    assert out.value is None


def test_invalid_router_handles_fail_cleanly():
    L, bogus = B.lib(), ctypes.c_void_p(0xdead0)
    for h in (bogus, None):
        assert L.moe_route(h, 1, P16, P16, P16, None, None, None) == B.MOE_ESTATE
        assert L.moe_route_backward(h, 1, P16, P16, P16, P16, None, P16, P16, None) == B.MOE_ESTATE
    assert L.moe_router_destroy(bogus) == B.MOE_ESTATE
    assert L.moe_router_destroy(None) == B.MOE_EINVAL
    assert L.moe_layer_set_router(bogus, None) == B.MOE_ESTATE
    assert L.moe_layer_set_router(None, bogus) == B.MOE_ESTATE


def test_layernorm_rejects_bad_args():
    L = B.lib()
    f = ctypes.c_float

    def fwd(h=P16, gain=None, bias=None, x=P16, type=0, T=4, d=64, eps=1e-5):
        return L.moe_layernorm(h, gain, bias, x, type, T, d, f(eps), None)

    for bad in [dict(h=None), dict(x=None), dict(type=2), dict(T=0), dict(d=0), dict(d=96),
                dict(d=16448), dict(eps=-1.0), dict(eps=float("nan")), dict(h=ODD), dict(x=ODD),
                dict(gain=ODD), dict(bias=ODD), dict(T=2097153)]:
        assert fwd(**bad) == B.MOE_EINVAL, bad

    def bwd(dx=P16, type=0, h=P16, gain=None, eps=1e-5, T=4, d=64, dh=P16, dg=P16, db=P16, ws=P16):
        return L.moe_layernorm_backward(dx, type, h, gain, f(eps), T, d, dh, 0, dg, db, ws, None)

    for bad in [dict(dx=None), dict(h=None), dict(dh=None), dict(type=3), dict(T=0), dict(d=96),
                dict(eps=-1.0), dict(ws=None), dict(ws=None, dg=None), dict(ws=None, db=None),
                dict(dx=ODD), dict(h=ODD), dict(gain=ODD), dict(dh=ODD), dict(dg=ODD),
                dict(db=ODD), dict(ws=ODD), dict(T=2097153)]:
        assert bwd(**bad) == B.MOE_EINVAL, bad


def test_layernorm_workspace_sizes():
    assert B.layernorm_workspace(1, 64) >= 2 * 64 * 4
    for T, d in [(1, 64), (200, 320), (8192, 4096), (100000, 16384)]:
        assert B.layernorm_workspace(T, d) % 256 == 0
    n = ctypes.c_int64()
    for T, d in [(0, 64), (4, 96), (4, 0), (4, 16448), (2097153, 64)]:
        assert B.lib().moe_layernorm_workspace(T, d, ctypes.byref(n)) == B.MOE_EINVAL
    assert B.lib().moe_layernorm_workspace(4, 64, None) == B.MOE_EINVAL


def test_binding_refuses_types_and_host_tensors():
    torch = pytest.importorskip("torch")
    h, x = torch.zeros((2, 64)), torch.zeros((2, 64), dtype=torch.float16)
    with pytest.raises(ValueError, match="device tensor"):
        B.layernorm(h, x)
    with pytest.raises(ValueError, match="two-dimensional"):
        B.layernorm([0.0], x)
    with pytest.raises(ValueError, match="two-dimensional"):
        B.layernorm(h[0], x)
    with pytest.raises(ValueError, match="float16 or torch.bfloat16"):
        B.MoeRouter(64, 4, 2, 8, x, dtype=torch.float32)
    with pytest.raises(ValueError, match="device tensor"):
        B.MoeRouter(64, 2, 2, 8, x)
    with pytest.raises(ValueError, match="needs a workspace"):
        B.layernorm_backward(x, h, h, d_gain=h[0], stream=1)
