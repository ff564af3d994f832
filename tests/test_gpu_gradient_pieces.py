"""Gradient lists around the pieces that a block takes (32 KB of a tensor: 16384
elements of 16 bits, 8192 of fp32) and around the eight vectors that a thread
loads at once, on and off the 16-byte grid.

Bounds: those of the list's other tests.  u = 2^-24; the norm is off by its own
rounding (squares are summed in 64 bits); the factor carries two roundings to
fp32, the product a third, and the tensor's type half a step (or half of its
smallest subnormal)."""
import numpy as np
import pytest

from oracle import experts_oracle as X

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

U = 2.0 ** -24
HALF = {torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8, torch.float32: 0.0}
TINY = {torch.float16: 2.0 ** -25, torch.bfloat16: 2.0 ** -134, torch.float32: 2.0 ** -150}
TYPES = pytest.mark.parametrize("dtype", list(HALF), ids=["f16", "bf16", "f32"])
PIECE = 1 << 15


@pytest.fixture(scope="module", autouse=True)
def _need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2411_01433_amd as P
    P.lib()
    yield


def _f64(t):
    return t.double().cpu().numpy()


def _check(before, outs, norm, max_norm):
    ref, _ = X.clip([_f64(g) for g in before], max_norm)
    assert abs(float(norm.item()) - ref) <= 1.001 * U * ref
    for g, o in zip(before, outs):
        want = _f64(g) * min(1.0, max_norm / (ref + 1e-6))
        assert (np.abs(_f64(o) - want) <= (3.01 * U + HALF[g.dtype]) * np.abs(want) + TINY[g.dtype]).all()


@TYPES
@pytest.mark.parametrize("shift", [0, 1, 5])
@pytest.mark.parametrize("place", ["in", "out", "out, off the grid of in"])
def test_sizes_around_a_piece(dtype, shift, place):
    import paper_2411_01433_amd as P
    per = PIECE // torch.finfo(dtype).bits * 8
    vec = 16 * 8 // torch.finfo(dtype).bits
    sizes = [per - vec, per - 1, per, per + 1, 2 * per, 2 * per + vec + 1, 7 * 256 * vec,
             7 * 256 * vec + 1, 8 * 256 * vec - 1, 5 * per - 3]
    g = torch.Generator().manual_seed(shift)
    hold = lambda n, k: torch.full((n + 16,), 7.0, dtype=dtype, device="cuda")[k:k + n]
    grads = []
    for n in sizes:
        t = hold(n, shift)
        t.copy_((0.1 * torch.randn(n, generator=g)).to(dtype))
        grads.append(t)
    outs = None if place == "in" else [hold(n, shift + (1 if "off" in place else 0)) for n in sizes]
    before = [t.clone() for t in grads]
    norm = torch.zeros(1, device="cuda")
    P.MoeGradients(grads, outs).clip(0.05, norm)
    _check(before, outs or grads, norm, 0.05)
    for t in grads + (outs or []):  # what lies around each is left as it was
        around = torch.empty(0, dtype=dtype, device="cuda").set_(t.untyped_storage())
        a, n = t.storage_offset(), t.numel()
        assert (around[:a] == 7.0).all() and (around[a + n:] == 7.0).all()
    if outs:
        assert all(torch.equal(a, b) for a, b in zip(grads, before))


@TYPES
def test_clip_is_norm_and_scale(dtype):
    """One call gives the bits of the two."""
    import paper_2411_01433_amd as P
    g = torch.Generator().manual_seed(1)
    grads = [(0.1 * torch.randn(n, generator=g)).to(dtype).cuda() for n in (3, 16384, 100001)]
    one, two = ([torch.empty_like(t) for t in grads] for _ in range(2))
    n1, n2 = torch.zeros(1, device="cuda"), torch.zeros(1, device="cuda")
    P.MoeGradients(grads, one).clip(0.3, n1)
    h = P.MoeGradients(grads, two)
    h.norm(n2)
    h.scale(0.3, n2)
    assert torch.equal(n1, n2) and all(torch.equal(a, b) for a, b in zip(one, two))
