"""The timed cases of perf/more_operators.py at small sizes: the framework's calls
run on what `prepare` gives, return what the plain form returns (paths, shapes,
types), whole numbers are equal, and both are as near to the 64-bit values as
the outputs' type and the sums allow.

Bounds.  u = 2^-24 is half a step of fp32.  Each output is a sum of at most n
products in fp32, off by 4 u sqrt(n) of the whole output's norm (the bound of the
grouped products' tests), rounded once to its type (half a step, and half of the
smallest subnormal of fp16).  The norm and the clipped gradients carry at most
four roundings to fp32 (norm, factor, product, type): n = 1 has room for five."""
import importlib.util
import os

import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

U = 2.0 ** -24
HALF = {torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8, torch.float32: U}
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

MX = {"kind": "mx_product", "T": 9, "d": 320, "f": 192, "E": 4, "K": 2}
CASES = [
    {"kind": "product", "type": "f16", "T": 5, "d": 256, "f": 448, "E": 8, "K": 2},
    {"kind": "backward", "type": "bf16", "T": 33, "d": 192, "f": 128, "E": 4, "K": 3},
    {"kind": "quantize", "type": "bf16", "rows": 3, "cols": 192},
    {"kind": "quantize", "type": "f16", "rows": 130, "cols": 64},
    {**MX, "type": "f16", "act": "16"}, {**MX, "type": "bf16", "act": "16"},
    {**MX, "type": "f16", "act": "4"}, {**MX, "type": "bf16", "act": "4", "T": 300},
    {"kind": "clip", "layers": 2, "d": 61, "E": 3, "f": 0, "experts": "f32", "clipped": True},
    {"kind": "clip", "layers": 1, "d": 64, "E": 3, "f": 37, "experts": "bf16", "clipped": True},
    {"kind": "clip", "layers": 1, "d": 64, "E": 3, "f": 37, "experts": "f16", "clipped": False},
]


@pytest.fixture(scope="module")
def cases():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    spec = importlib.util.spec_from_file_location("timed_cases", os.path.join(ROOT, "perf", "more_operators.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def _leaves(v, path=""):
    if isinstance(v, dict):
        return [x for k in sorted(v) for x in _leaves(v[k], f"{path}.{k}")]
    if isinstance(v, list):
        return [x for i, t in enumerate(v) for x in _leaves(t, f"{path}[{i}]")]
    return [(path, v)]


def _near(got, ref, n):
    small = 2.0 ** -25 * ref.numel() ** 0.5 if got.dtype is torch.float16 else 0.0
    err = (got.double() - ref).norm()
    assert float(err) <= (HALF[got.dtype] + 4 * U * n ** 0.5) * float(ref.norm()) + small


@pytest.mark.parametrize("case", CASES, ids=lambda c: "-".join(str(v) for v in c.values()))
def test_both_sides(cases, case):
    sides = []
    for own in (False, True):
        cases.own = own
        s = cases.prepare(case, 3)
        cases.run(s)
        sides.append(_leaves(cases.run(s)))  # (the second pass on a state, as the first)
    cases.own = False
    exact = dict(_leaves(cases.exact(case, 3)))
    n = {"product": 256, "backward": 128, "mx_product": 320}.get(case["kind"], 1)
    assert len(sides[0]) == len(sides[1]) and sides[0]
    for (path, a), (path2, b) in zip(*sides):
        assert (path, a.shape, a.dtype) == (path2, b.shape, b.dtype)
        if not a.is_floating_point():
            assert torch.equal(a, b), path
        if exact[path] is not None:
            _near(a, exact[path], n)
            _near(b, exact[path], n)


def test_every_listed_and_drawn_case_has_work(cases):
    import random
    rng = random.Random(1)
    for case in cases.listed() + [cases.draw(rng) for _ in range(20)]:
        w = cases.work(case)
        assert w["bytes"] > 0 and w["flops"] > 0
