"""What follows the routing of an MoE layer when its experts are tuned or
served in 4 bits, as timed cases: products grouped by expert with their
backward pass, the microscaled 4-bit quantiser and its products, and the norm
and clipping of the gradients.  `run` computes an operator in its plain form
(elementary torch operations), or, with `own` set, through this package's
entry points.

Rows of x are sorted by expert, `count[e]` of them for expert e.

Product      y[r] = W[e(r)] x[r], W [E, f, d]
Backward     d_x[r] = W[e(r)]^T d_y[r];  d_W[e] = sum over e's rows of d_y[r] x[r]^T (fp32)
Quantise     per 32 columns: scale 2^e, e = floor(log2 max|v|) - 2 (at least
             -127), codes the nearest of +-{0, .5, 1, 1.5, 2, 3, 4, 6} to v / 2^e
             (ties to the even code, beyond 6 to 6); two codes a byte, the lower
             column in the lower half; the scale as the byte e + 127
MX product   the grouped product with W in that format; x of 16 bits (W's
             values in x's type) or quantised in the call
Clip         norm = sqrt(sum of all squares); out = g min(1, c / (norm + 1e-6))

Shapes are this repository's layers (d_model 4096; d_ff 14336 with 8 experts,
6400 with 16, top-2) and generic ones of more, smaller experts.  Hidden states
are N(0, 1), weights N(0, 0.02), as everywhere in this repository.
"""
from __future__ import annotations

import math

import torch

own = False
DEV = "cuda"
W_STD = 0.02
CLIP_EPS = 1e-6
TYPES = {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}


def listed():
    mixtral = {"d": 4096, "f": 14336, "E": 8, "K": 2}
    phi = {"d": 4096, "f": 6400, "E": 16, "K": 2}
    small = {"d": 2048, "f": 1472, "E": 60, "K": 4}
    return [
        # one sequence being decoded: two experts' weights are read for one row each
        {"name": "product_t1_e8", "kind": "product", "type": "f16", "T": 1, **mixtral},
        # an odd prompt on many small experts: about 90 rows each
        {"name": "product_t1337_e60_bf16", "kind": "product", "type": "bf16", "T": 1337, **small},
        # a training step's forward, or the largest prefill
        {"name": "product_t8192_e16", "kind": "product", "type": "f16", "T": 8192, **phi},
        # tuning many small experts on one odd prompt
        {"name": "backward_t1337_e60_bf16", "kind": "backward", "type": "bf16", "T": 1337, **small},
        # a training step's backward
        {"name": "backward_t4096_e16", "kind": "backward", "type": "f16", "T": 4096, **phi},
        # the activations of a decode batch
        {"name": "quantize_32x4096_bf16", "kind": "quantize", "type": "bf16", "rows": 32,
         "cols": 4096},
        # one matrix of an expert enters the 4-bit cache
        {"name": "quantize_14336x4096", "kind": "quantize", "type": "f16", "rows": 14336,
         "cols": 4096},
        # one sequence being decoded from 4-bit weights
        {"name": "mx_product_t1_e8", "kind": "mx_product", "type": "f16", "act": "16", "T": 1,
         **mixtral},
        # a prompt on 4-bit weights, activations kept at 16 bits
        {"name": "mx_product_t512_e16_bf16", "kind": "mx_product", "type": "bf16", "act": "16",
         "T": 512, **phi},
        # a long prompt with activations in 4 bits too
        {"name": "mx_product_t4096_e16_4bit", "kind": "mx_product", "type": "f16", "act": "4",
         "T": 4096, **phi},
        # tuning the gates and norms of a stack: many small tensors
        {"name": "clip_16_layers_gates", "kind": "clip", "layers": 16, "d": 4096, "E": 8, "f": 0,
         "experts": "f32", "clipped": True},
        # tuning a layer's experts: gradients of 0.8 GB
        {"name": "clip_experts_e8", "kind": "clip", "layers": 1, "d": 2048, "E": 8, "f": 4096,
         "experts": "f32", "clipped": True},
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["product", "product", "backward", "backward", "quantize", "mx_product",
                       "mx_product", "mx_product", "clip"])
    if kind == "quantize":
        return {"kind": kind, "type": rng.choice(["f16", "bf16"]),
                "rows": _log_int(rng, 1, 14336), "cols": 64 * _log_int(rng, 1, 64)}
    E = rng.choice([1, 2, 4, 6, 8, 16, 40, 60, 64, 96, 128, 256])
    d = 64 * _log_int(rng, 4, 64)
    if kind == "clip":
        layers = rng.randint(1, 9)
        f = rng.choice([0, rng.randint(1, 2000)])
        while layers * 3 * E * f * d > 190_000_000:
            f //= 2
        return {"kind": kind, "layers": layers, "d": d - rng.randint(0, 3), "E": E, "f": f,
                "experts": rng.choice(["f32", "f32", "bf16", "f16"]), "clipped": rng.random() < 0.7}
    c = {"kind": kind, "type": rng.choice(["f16", "bf16"])}
    if kind == "mx_product":
        c["act"] = rng.choice(["16", "4"])
    f = 64 * _log_int(rng, 6, 224)
    while E * f * d > 400_000_000:
        f, E = max(64, f // 128 * 64), max(1, E // 2)
    K = rng.randint(1, min(E, 8))
    T = _log_int(rng, 1, 8192)
    most = 16384 * 6400 * 4096 if kind == "product" else 8192 * 6400 * 4096
    while T * K * f * d > most:
        T = T * 2 // 3
    return {**c, "T": T, "d": d, "f": f, "E": E, "K": K}


# ---- inputs ------------------------------------------------------------------

def _normal(g, shape, std=1.0, dtype=torch.float32):
    return torch.empty(shape, device=DEV, dtype=dtype).normal_(0.0, std, generator=g)


def _counts(case, g):
    """Rows of each expert: T tokens take K different experts each, some experts more often."""
    T, E, K = case["T"], case["E"], case["K"]
    lg = _normal(g, (1, E), 0.5) - torch.log(-torch.log(torch.rand((T, E), device=DEV, generator=g)
                                                        .clamp(1e-6, 1 - 1e-6)))
    return torch.bincount(torch.topk(lg, K, dim=-1).indices.view(-1), minlength=E).int()


def _mx(v):
    """(values / scale, magnitudes and signs apart; exponents) of the 4-bit format, in fp32."""
    b = v.float().view(*v.shape[:-1], -1, 32)
    top = b.abs().amax(-1)
    e = torch.where(top > 0, torch.frexp(top).exponent - 3, -127).clamp(min=-127)
    # (in two steps: a scale below 2^-126 has no fp32 reciprocal)
    h = -e // 2
    a = torch.ldexp(torch.ldexp(b, h[..., None]), (-e - h)[..., None])
    m = a.abs()
    step = 0.5 + 0.5 * (m >= 2) + (m >= 4)
    return ((m / step).round() * step).clamp(max=6.0), torch.signbit(a), e


def _mx_pack(v):
    """codes [.., cols / 2] and scales [.., cols / 32] (uint8) of v."""
    m, neg, e = _mx(v)
    k = torch.where(m < 2, 2 * m, torch.where(m < 4, m + 2, m / 2 + 4)).to(torch.uint8)
    k = (k + 8 * neg).view(*v.shape[:-1], -1, 2)
    return k[..., 0] + 16 * k[..., 1], (e + 127).to(torch.uint8)


def _mx_unpack(codes, scales, dtype):
    """The values of codes and scales."""
    lut = torch.tensor([0, .5, 1, 1.5, 2, 3, 4, 6, 0, -.5, -1, -1.5, -2, -3, -4, -6], device=DEV,
                       dtype=dtype)
    k = torch.stack((codes & 15, codes >> 4), -1).int()
    v = lut[k].view(*scales.shape, 32)
    e = scales.int() - 127
    h = e // 2
    return torch.ldexp(torch.ldexp(v, h[..., None]), (e - h)[..., None]).flatten(-2)


def _inputs(case, seed):
    g = torch.Generator(device=DEV).manual_seed(seed)
    kind = case["kind"]
    if kind == "quantize":
        # rows of different size, as channels and tokens have
        v = _normal(g, (case["rows"], case["cols"])) * torch.exp(_normal(g, (case["rows"], 1)))
        return {"v": v.to(TYPES[case["type"]])}
    if kind == "clip":
        E, d, f = case["E"], case["d"], case["f"]
        grads = []
        for _ in range(case["layers"]):
            grads += [_normal(g, (E, d), 0.02), _normal(g, (d,), 0.1), _normal(g, (d,), 0.1)]
            if f:
                grads += [_normal(g, s, 0.01, TYPES[case["experts"]])
                          for s in ((E, f, d), (E, f, d), (E, d, f))]
        return {"g": grads, "max_norm": 1.0 if case["clipped"] else 1e6}
    t, d, f, E = TYPES[case["type"]], case["d"], case["f"], case["E"]
    R = case["T"] * case["K"]
    s = {"count": _counts(case, g), "x": _normal(g, (R, d), 1.0, t)}
    w = _normal(g, (E, f, d), W_STD, t)
    if kind == "mx_product":
        s["codes"], s["scales"] = _mx_pack(w)
    else:
        s["w"] = w
    if kind == "backward":
        s["dy"] = _normal(g, (R, f), 0.05, t)
    return s


def _plan(s, R):
    """The rows as one block per expert that has any, all as long as the longest."""
    count = s["count"].long()
    s["act"] = torch.nonzero(count).view(-1)
    n, first = count[s["act"]], (count.cumsum(0) - count)[s["act"]]
    at = torch.arange(int(n.max()), device=DEV)
    s["held"] = at < n[:, None]
    s["row"] = torch.where(s["held"], first[:, None] + at, R)  # row R: zeros


def prepare(case, seed):
    s = _inputs(case, seed)
    s["case"] = case
    kind = case["kind"]
    if kind == "quantize":
        r, c = case["rows"], case["cols"]
        s["codes"] = torch.empty((r, c // 2), dtype=torch.uint8, device=DEV)
        s["scales"] = torch.empty((r, c // 32), dtype=torch.uint8, device=DEV)
        s["values"] = torch.empty_like(s["v"])
        return s
    if kind == "clip":
        s["out"] = [torch.empty_like(g) for g in s["g"]]
        s["norm"] = torch.empty(1, device=DEV)
        if own:
            import paper_2411_01433_amd as P
            s["grads"] = P.MoeGradients(s["g"], s["out"])
        return s
    t, d, f, E = TYPES[case["type"]], case["d"], case["f"], case["E"]
    R = case["T"] * case["K"]
    _plan(s, R)
    if kind == "backward":
        s["d_x"] = torch.empty((R, d), dtype=t, device=DEV)
        s["d_w"] = torch.empty((E, f, d), device=DEV)
    else:
        s["y"] = torch.empty((R, f), dtype=t, device=DEV)
        if case.get("act") == "4":
            s["x_codes"] = torch.empty((R, d // 2), dtype=torch.uint8, device=DEV)
            s["x_scales"] = torch.empty((R, d // 32), dtype=torch.uint8, device=DEV)
    return s


# ---- one pass ----------------------------------------------------------------

def run(s):
    return _run_own(s) if own else _run_plain(s)


def _w_codes(s):
    """W's codes as the bytes that the calls take: laid out once for a state, as a program that
    serves them keeps its weights (the plain form's are whole numbers of 64 bits)."""
    if "w_codes" not in s:
        s["w_codes"] = s["codes"].to(torch.uint8)
    return s["w_codes"]


def _run_own(s):
    import paper_2411_01433_amd as P
    kind = s["case"]["kind"]
    if kind == "product":
        P.grouped_product(s["x"], s["w"], s["y"], s["count"])
        return {"y": s["y"]}
    if kind == "backward":
        P.grouped_product_backward(s["dy"], s["x"], s["w"], s["count"], s["d_x"], s["d_w"])
        return {"x": s["d_x"], "w": s["d_w"]}
    if kind == "quantize":
        P.mx_quantize(s["v"], s["codes"], s["scales"], s["values"])
        # (the codes in the type in which the plain form has them, so that they compare: a copy
        # of 8 bytes for each pair, which no program needs, and which is timed with the call)
        return {"codes": s["codes"].long(), "scales": s["scales"], "values": s["values"]}
    if kind == "mx_product":
        w = _w_codes(s)
        if s["case"]["act"] == "4":
            P.mx_quantize(s["x"], s["x_codes"], s["x_scales"])
            P.mx_product(s["x_codes"], w, s["scales"], s["y"], s["count"], s["x_scales"])
        else:
            P.mx_product(s["x"], w, s["scales"], s["y"], s["count"])
        return {"y": s["y"]}
    s["grads"].clip(s["max_norm"], s["norm"])
    return {"norm": s["norm"], "out": s["out"]}


def _blocks(v, s):
    """Rows of v (fp32) as the plan's blocks, zeros behind an expert's last row."""
    return torch.cat((v, v.new_zeros((1, v.shape[1]))))[s["row"]]


def _run_plain(s):
    case = s["case"]
    kind = case["kind"]
    if kind == "quantize":
        m, neg, e = _mx(s["v"])
        codes, scales = _mx_pack(s["v"])
        h = e // 2
        v = torch.ldexp(torch.ldexp(torch.where(neg, -m, m), h[..., None]), (e - h)[..., None])
        return {"codes": codes, "scales": scales, "values": v.flatten(-2).to(s["v"].dtype)}
    if kind == "clip":
        # (the sum in 64 bits: it is long)
        sq = [(g.float() * g.float()).sum(dtype=torch.float64) for g in s["g"]]
        norm = torch.sqrt(torch.stack(sq).sum())
        c = (s["max_norm"] / (norm + CLIP_EPS)).clamp(max=1.0).float()
        return {"norm": norm.float().view(1), "out": [(g.float() * c).to(g.dtype) for g in s["g"]]}
    t = TYPES[case["type"]]
    if kind == "backward":
        dy = _blocks(s["dy"].float(), s)
        dx = torch.bmm(dy, s["w"][s["act"]].float())[s["held"]]
        dw = torch.zeros(s["w"].shape, device=DEV)
        dw[s["act"]] = torch.bmm(dy.transpose(1, 2), _blocks(s["x"].float(), s))
        return {"x": dx.to(t), "w": dw}
    if kind == "product":
        x, w = s["x"].float(), s["w"][s["act"]].float()
    else:
        w = _mx_unpack(s["codes"][s["act"]], s["scales"][s["act"]], torch.float32).to(t).float()
        x = s["x"].float()
        if case["act"] == "4":
            x = _mx_unpack(*_mx_pack(s["x"]), torch.float32)
    return {"y": torch.bmm(_blocks(x, s), w.transpose(1, 2))[s["held"]].to(t)}


# ---- what a pass cannot do without -----------------------------------------------

def work(case):
    kind = case["kind"]
    if kind == "quantize":
        n = case["rows"] * case["cols"]
        return {"bytes": n * (2 + 0.5 + 1 / 32 + 2), "flops": 3.0 * n}
    if kind == "clip":
        small = case["layers"] * (case["E"] + 2) * case["d"]
        big = case["layers"] * 3 * case["E"] * case["f"] * case["d"]
        size = 4 if case["experts"] == "f32" else 2
        return {"bytes": 2.0 * (4 * small + size * big), "flops": 3.0 * (small + big)}
    d, f, E, K = case["d"], case["f"], case["E"], case["K"]
    R = case["T"] * K
    # distinct experts that T independent tokens are expected to select
    experts = E * (1.0 - (1.0 - K / E) ** case["T"]) if K < E else E
    if kind == "backward":
        return {"bytes": experts * f * d * 2 + R * (2 * d + f) * 2 + E * f * d * 4.0,
                "flops": 4.0 * R * f * d}
    per = 2.0 if kind == "product" else 0.5 + 1 / 32
    return {"bytes": experts * f * d * per + R * (d + f) * 2, "flops": 2.0 * R * f * d}


# ---- the same in 64 bits -----------------------------------------------------------

GRID = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]


def _nearest(v):
    """The 4-bit format's values of v, in 64 bits."""
    b = v.double().reshape(v.shape[0], -1, 32)
    top = b.abs().amax(-1, keepdim=True)
    p = torch.exp2(torch.floor(torch.log2(top.clamp_min(2.0 ** -125))) - 2)
    a = (b / p).abs()
    best = torch.zeros_like(a)
    off = a.clone()  # how far 0 is
    for k, value in enumerate(GRID[1:], 1):
        d = (a - value).abs()
        near = (d < off) | ((d == off) & (k % 2 == 0))
        best, off = torch.where(near, value, best), torch.where(near, d, off)
    return (torch.sign(b) * best * p).reshape(v.shape)


def _values(codes, scales):
    """What codes and scales stand for, in 64 bits."""
    k = torch.stack((codes % 16, codes // 16), -1).flatten(-2)
    v = torch.tensor(GRID, dtype=torch.float64, device=DEV)[(k % 8).long()] * (1.0 - 2.0 * (k >= 8))
    p = torch.exp2(scales.double() - 127.0)
    return (v.view(*p.shape, 32) * p[..., None]).flatten(-2)


def exact(case, seed):
    kind = case["kind"]
    # products in 64 bits take a second for 5e13 operations
    if kind not in ("quantize", "clip") and work(case)["flops"] > 9e14:
        return None
    s = _inputs(case, seed)
    if kind == "quantize":
        return {"codes": None, "scales": None, "values": _nearest(s["v"])}
    if kind == "clip":
        norm = math.sqrt(math.fsum(float(g.double().square().sum()) for g in s["g"]))
        c = min(1.0, s["max_norm"] / (norm + CLIP_EPS))
        return {"norm": torch.tensor([norm], dtype=torch.float64, device=DEV),
                "out": [c * g.double() for g in s["g"]]}
    x, at = s["x"].double(), 0
    if case.get("act") == "4":
        x = _nearest(s["x"])
    y = torch.empty((x.shape[0], case["d" if kind == "backward" else "f"]), dtype=torch.float64,
                    device=DEV)
    dw = torch.zeros((case["E"], case["f"], case["d"]), dtype=torch.float64,
                     device=DEV) if kind == "backward" else None
    for e, n in enumerate(s["count"].tolist()):
        rows = slice(at, at + n)
        at += n
        if n == 0:
            continue
        if kind == "mx_product":
            w = _values(s["codes"][e], s["scales"][e])
        else:
            w = s["w"][e].double()
        if kind == "backward":
            dy = s["dy"][rows].double()
            y[rows] = dy @ w
            dw[e] = dy.T @ x[rows]
        else:
            y[rows] = x[rows] @ w.T
    return {"x": y, "w": dw} if kind == "backward" else {"y": y}
