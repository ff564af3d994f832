"""The training and serving front of an MoE layer, as timed cases: the layer
norm of the residual stream and the routing of its rows to experts, each with
its backward pass.  `run` computes an operator in its plain form (elementary
torch operations), or, with `own` set, through this package's entry points.

Layer norm   x = (h - mean h) / sqrt(var h + eps) * gain + bias, per row of h
Routing      l = x Wg^T;  s = sigmoid(l) or softmax(l) over the experts;
             key = s + b (or l where there is no bias b); experts in groups:
             a group's score is the sum of its best one or two keys (of
             scores s where there is no bias), and the best groups stay; the
             top_k experts of the largest keys, ties to the lower index;
             weights: scale * s, or scale * s / (sum of the selected s)
Backward     of the weights and of the logits to x and Wg; the bias and the
             selection have no gradient

Shapes are this repository's layers (d_model 4096; 8 and 16 experts, top-2)
and generic ones of more, smaller experts.  Hidden states are N(0, 1), weights
N(0, 0.02), as everywhere in this repository.
"""
from __future__ import annotations

import math

import torch

own = False
DEV = "cuda"
W_STD = 0.02
EPS = 1e-5
TYPES = {"f16": torch.float16, "bf16": torch.bfloat16}


def listed():
    route = {"score": "sigmoid", "bias": True, "groups": 8, "top_groups": 4, "best": 2,
             "renorm": True, "scale": 2.5}
    plain = {"score": "softmax", "bias": False, "groups": 1, "top_groups": 1, "best": 1,
             "renorm": True, "scale": 1.0}
    return [
        # one sequence being decoded on a layer of 16 experts: latency only
        {"name": "route_t1_e16", "kind": "route", "type": "f16", "T": 1, "d": 4096, "E": 16,
         "K": 2, **plain, "train": False},
        # a decode batch on a layer of many small experts, balanced by a bias and routed by groups
        {"name": "route_t32_e256_groups", "kind": "route", "type": "f16", "T": 32, "d": 4096,
         "E": 256, "K": 8, **route, "train": False},
        # an odd prompt, weights kept as they are in the softmax over all experts
        {"name": "route_t1337_e60_bf16", "kind": "route", "type": "bf16", "T": 1337, "d": 2048,
         "E": 60, "K": 4, **plain, "renorm": False, "train": True},
        # a training step's forward: logits and the experts' loads are kept
        {"name": "route_t8192_e256_groups", "kind": "route", "type": "f16", "T": 8192, "d": 4096,
         "E": 256, "K": 8, **route, "train": True},
        # tuning the gate of a layer of 8 experts on a short prompt
        {"name": "route_backward_t512_e8", "kind": "route_backward", "type": "f16", "T": 512,
         "d": 4096, "E": 8, "K": 2, **plain, "aux": False},
        # odd sizes; losses on the logits themselves (balance, magnitude) beside the weights'
        {"name": "route_backward_t1337_e60_bf16", "kind": "route_backward", "type": "bf16",
         "T": 1337, "d": 2048, "E": 60, "K": 4, **plain, "renorm": False, "aux": True},
        # a training step's backward on many experts
        {"name": "route_backward_t8192_e256", "kind": "route_backward", "type": "f16", "T": 8192,
         "d": 4096, "E": 256, "K": 8, **route, "aux": False},
        # the norm before a layer for one decoded token: latency only
        {"name": "layernorm_t1", "kind": "layernorm", "type": "f16", "T": 1, "d": 4096},
        # the norm of a long prompt or a training step
        {"name": "layernorm_t8192", "kind": "layernorm", "type": "f16", "T": 8192, "d": 4096},
        # a small, odd layer in training
        {"name": "layernorm_backward_t200_bf16", "kind": "layernorm_backward", "type": "bf16",
         "T": 200, "d": 320},
        # tuning on one prompt
        {"name": "layernorm_backward_t512", "kind": "layernorm_backward", "type": "f16", "T": 512,
         "d": 4096},
        # a training step's backward
        {"name": "layernorm_backward_t8192", "kind": "layernorm_backward", "type": "f16",
         "T": 8192, "d": 4096},
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["route", "route", "route", "route_backward", "route_backward", "layernorm",
                       "layernorm_backward"])
    d = 64 * _log_int(rng, 4, 128)
    c = {"kind": kind, "type": rng.choice(["f16", "bf16"]), "d": d,
         "T": _log_int(rng, 1, min(8192, 8192 * 4096 // d))}
    if kind.startswith("layernorm"):
        return c
    E = rng.choice([4, 6, 8, 16, 40, 60, 64, 96, 128, 160, 256])
    c["E"] = E
    c["K"] = rng.randint(1, min(E, rng.choice([2, 4, 8])))
    c["score"] = rng.choice(["sigmoid", "softmax"])
    c["bias"] = rng.random() < 0.5
    c["groups"] = rng.choice([g for g in (1, 1, 2, 4, 8) if E % g == 0])
    size = E // c["groups"]
    c["top_groups"] = rng.randint(min(c["groups"], -(-c["K"] // size)), c["groups"])
    c["best"] = rng.choice([1, 2])
    c["renorm"] = rng.random() < 0.6
    c["scale"] = rng.choice([1.0, 2.5])
    if kind == "route":
        c["train"] = rng.random() < 0.5
    else:
        # (one renormalised weight is the scale itself and has no gradient)
        c["aux"] = rng.random() < 0.5 or (c["renorm"] and c["K"] == 1)
    return c


# ---- inputs ------------------------------------------------------------------

def _normal(g, shape, std=1.0, dtype=torch.float32):
    return torch.empty(shape, device=DEV).normal_(0.0, std, generator=g).to(dtype)


def _inputs(case, seed):
    g = torch.Generator(device=DEV).manual_seed(seed)
    T, d, t = case["T"], case["d"], TYPES[case["type"]]
    if case["kind"].startswith("layernorm"):
        # a residual stream: an offset per row, some channels far larger than the rest
        h = _normal(g, (T, d)) + 0.5 * _normal(g, (T, 1))
        h[:, ::97] *= 8.0
        s = {"h": h, "gain": 1.0 + _normal(g, (d,), 0.1), "bias": _normal(g, (d,), 0.1)}
        if case["kind"] == "layernorm_backward":
            s["dx"] = _normal(g, (T, d), 0.01, t)
        return s
    E, K = case["E"], case["K"]
    s = {"x": _normal(g, (T, d), 1.0, t), "wg": _normal(g, (E, d), W_STD, t)}
    # what steers the balance moves the scores by a few per cent of their range
    s["b"] = _normal(g, (E,), 0.02 if case["score"] == "sigmoid" else 0.2 / E) if case["bias"] else None
    if case["kind"] == "route_backward":
        # what the forward pass left behind, and the gradients that arrive
        s["logits"] = (s["x"].double() @ s["wg"].double().T).float()
        s["idx"] = _select(case, s["logits"].double(), s["b"])
        # (fp16 training scales its loss, so that gradients stay in range)
        s["dw"] = _normal(g, (T, K))
        s["dl"] = _normal(g, (T, E), 0.01) if case["aux"] else None
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    s["case"] = case
    T, d, t = case["T"], case["d"], TYPES[case["type"]]
    kind = case["kind"]
    if kind == "layernorm":
        s["x"] = torch.empty((T, d), dtype=t, device=DEV)
        return s
    if kind == "layernorm_backward":
        s["d_h"] = torch.empty((T, d), device=DEV)
        s["d_gain"], s["d_bias"] = torch.empty(d, device=DEV), torch.empty(d, device=DEV)
        if own:
            import paper_2411_01433_amd as P
            s["ws"] = torch.empty(P.layernorm_workspace(T, d), dtype=torch.uint8, device=DEV)
        return s
    E, K = case["E"], case["K"]
    if kind == "route":
        s["idx"] = torch.empty((T, K), dtype=torch.int32, device=DEV)
        s["w"] = torch.empty((T, K), device=DEV)
        s["logits"] = torch.empty((T, E), device=DEV) if case["train"] else None
        s["count"] = torch.empty(E, dtype=torch.int32, device=DEV) if case["train"] else None
    else:
        s["d_x"] = torch.empty((T, d), dtype=t, device=DEV)
        s["d_wg"] = torch.empty((E, d), device=DEV)
    if own:
        import paper_2411_01433_amd as P
        s["router"] = P.MoeRouter(
            d, E, K, T, s["wg"], s["b"], dtype=t,
            score=P.SCORE_SIGMOID if case["score"] == "sigmoid" else P.SCORE_SOFTMAX,
            n_groups=case["groups"], top_groups=case["top_groups"], group_best=case["best"],
            renormalize=case["renorm"], scale=case["scale"], backward=kind == "route_backward")
    return s


# ---- one pass ----------------------------------------------------------------

def run(s):
    return _run_own(s) if own else _run_plain(s)


def _run_own(s):
    import paper_2411_01433_amd as P
    kind = s["case"]["kind"]
    if kind == "layernorm":
        P.layernorm(s["h"], s["x"], s["gain"], s["bias"], EPS)
        return {"x": s["x"]}
    if kind == "layernorm_backward":
        P.layernorm_backward(s["dx"], s["h"], s["d_h"], s["gain"], s["d_gain"], s["d_bias"], EPS,
                             workspace=s["ws"])
        return {"h": s["d_h"], "gain": s["d_gain"], "bias": s["d_bias"]}
    if kind == "route":
        s["router"].route(s["x"], s["idx"], s["w"], s["logits"], s["count"])
        return {"idx": s["idx"], "w": s["w"], "logits": s["logits"], "count": s["count"]}
    s["router"].backward(s["x"], s["logits"], s["idx"], s["dw"], s["d_x"], s["d_wg"], s["dl"])
    return {"x": s["d_x"], "wg": s["d_wg"]}


def _select(case, lg, b):
    """The selected experts [T, K] (int32) by logits in 64 bits."""
    T, E, G = lg.shape[0], case["E"], case["groups"]
    s = torch.sigmoid(lg) if case["score"] == "sigmoid" else torch.softmax(lg, -1)
    key = lg if b is None else s + b.double()
    if G > 1:
        best = min(case["best"], E // G)
        score = (s if b is None else key).view(T, G, E // G)
        score = torch.sort(score, dim=-1, descending=True).values[..., :best].sum(-1)
        at = torch.sort(score, dim=-1, descending=True, stable=True).indices[:, :case["top_groups"]]
        keep = torch.zeros((T, G), dtype=torch.bool, device=lg.device).scatter_(1, at, True)
        key = key.masked_fill(~keep.repeat_interleave(E // G, 1), -math.inf)
    return torch.sort(key, dim=-1, descending=True, stable=True).indices[:, :case["K"]].int()


def _run_plain(s):
    case = s["case"]
    kind, t = case["kind"], TYPES[case["type"]]
    if kind.startswith("layernorm"):
        h = s["h"]
        c = h - h.mean(-1, keepdim=True)
        r = torch.rsqrt((c * c).mean(-1, keepdim=True) + EPS)
        n = c * r
        if kind == "layernorm":
            return {"x": (n * s["gain"] + s["bias"]).to(t)}
        dx = s["dx"].float()
        dn = dx * s["gain"]
        d_h = r * (dn - dn.mean(-1, keepdim=True) - n * (dn * n).mean(-1, keepdim=True))
        return {"h": d_h, "gain": (dx * n).sum(0), "bias": dx.sum(0)}
    if kind == "route":
        # in 64 bits: which of two near scores is larger decides what is selected
        lg = s["x"].double() @ s["wg"].double().T
        idx = _select(case, lg, s["b"])
        sc = torch.sigmoid(lg) if case["score"] == "sigmoid" else torch.softmax(lg, -1)
        w = torch.gather(sc, 1, idx.long())
        if case["renorm"]:
            w = w / w.sum(-1, keepdim=True)
        out = {"idx": idx, "w": (case["scale"] * w).float(), "logits": None, "count": None}
        if case["train"]:
            out["logits"] = lg.float()
            out["count"] = torch.bincount(idx.view(-1), minlength=case["E"]).int()
        return out
    lg, idx, dw = s["logits"], s["idx"].long(), case["scale"] * s["dw"]
    sig = case["score"] == "sigmoid"
    if case["renorm"]:
        v = torch.gather(torch.sigmoid(lg) if sig else torch.softmax(lg, -1), 1, idx)
        p = v / v.sum(-1, keepdim=True)
        g = p * (dw - (dw * p).sum(-1, keepdim=True)) * ((1 - v) if sig else 1.0)
        d_l = torch.zeros_like(lg).scatter_(1, idx, g)
    elif sig:
        v = torch.sigmoid(torch.gather(lg, 1, idx))
        d_l = torch.zeros_like(lg).scatter_(1, idx, dw * v * (1 - v))
    else:
        p = torch.softmax(lg, -1)
        d_p = torch.zeros_like(lg).scatter_(1, idx, dw)
        d_l = p * (d_p - (p * d_p).sum(-1, keepdim=True))
    if s["dl"] is not None:
        d_l = d_l + s["dl"]
    return {"x": (d_l @ s["wg"].float()).to(t), "wg": d_l.T @ s["x"].float()}


# ---- what a pass cannot do without ---------------------------------------------

def work(case):
    T, d = case["T"], case["d"]
    kind = case["kind"]
    if kind == "layernorm":
        return {"bytes": T * d * 6.0 + 8 * d, "flops": 9.0 * T * d}
    if kind == "layernorm_backward":
        return {"bytes": T * d * 10.0 + 12 * d, "flops": 18.0 * T * d}
    E, K = case["E"], case["K"]
    n = T * d * 2.0 + E * d * 2 + T * K * 8
    if kind == "route":
        return {"bytes": n + (T * E * 4 + E * 4 if case["train"] else 0), "flops": 2.0 * T * E * d}
    return {"bytes": n + T * d * 2 + E * d * 4 + T * E * (8 if case["aux"] else 4),
            "flops": 4.0 * T * E * d}


# ---- the same in 64 bits, from the definitions ----------------------------------

def _first_of_max(v):
    """(largest value, lowest index that has it) along the last axis."""
    top = v.max(-1, keepdim=True).values
    n = torch.arange(v.shape[-1], device=v.device).expand_as(v)
    return top, torch.where(v == top, n, v.shape[-1]).min(-1, keepdim=True).values


def exact(case, seed):
    s = _inputs(case, seed)
    kind = case["kind"]
    if kind.startswith("layernorm"):
        h, gain = s["h"].double(), s["gain"].double()
        sigma = (h.var(-1, unbiased=False, keepdim=True) + EPS).sqrt()
        n = (h - h.mean(-1, keepdim=True)) / sigma
        if kind == "layernorm":
            return {"x": gain * n + s["bias"].double()}
        dx = s["dx"].double()
        a = dx * gain
        rows = a - (a.sum(-1, keepdim=True) + n * (a * n).sum(-1, keepdim=True)) / case["d"]
        return {"h": rows / sigma, "gain": (dx * n).sum(0), "bias": dx.sum(0)}
    E, K, G, sc = case["E"], case["K"], case["groups"], case["scale"]
    x, wg = s["x"].double(), s["wg"].double()
    lg = x.matmul(wg.t()) if kind == "route" else s["logits"].double()
    if case["score"] == "sigmoid":
        score = 1.0 / (1.0 + torch.exp(-lg))
    else:
        score = torch.exp(lg - torch.logsumexp(lg, -1, keepdim=True))
    if kind == "route":
        key = lg if s["b"] is None else score + s["b"].double()
        if G > 1:
            left = (score if s["b"] is None else key).reshape(-1, G, E // G).clone()
            total = torch.zeros(left.shape[:2], dtype=torch.float64, device=x.device)
            for _ in range(min(case["best"], E // G)):
                top, at = _first_of_max(left)
                total += top[..., 0]
                left.scatter_(-1, at, -math.inf)
            kept = torch.full_like(total, -math.inf)
            for _ in range(case["top_groups"]):
                _, at = _first_of_max(total)
                kept.scatter_(-1, at, 0.0)
                total.scatter_(-1, at, -math.inf)
            key = key + kept.repeat_interleave(E // G, -1)
        else:
            key = key.clone()
        picked = []
        for _ in range(K):
            _, at = _first_of_max(key)
            picked.append(at)
            key.scatter_(-1, at, -math.inf)
        idx = torch.cat(picked, -1)
        w = score.gather(-1, idx)
        w = sc * (w / w.sum(-1, keepdim=True) if case["renorm"] else w)
        out = {"idx": idx.int(), "w": w, "logits": None, "count": None}
        if case["train"]:
            out["logits"] = lg
            out["count"] = (idx[..., None] == torch.arange(E, device=x.device)).sum((0, 1)).int()
        return out
    on = torch.zeros_like(lg).scatter_(-1, s["idx"].long(), 1.0)
    up = sc * torch.zeros_like(lg).scatter_(-1, s["idx"].long(), s["dw"].double())
    slope = 1.0 - score  # d log(score) / d logit: of a sigmoid
    if case["renorm"]:
        share = on * score / (on * score).sum(-1, keepdim=True)
        d_l = share * (up - (up * share).sum(-1, keepdim=True))
        d_l = d_l * slope if case["score"] == "sigmoid" else d_l
    elif case["score"] == "sigmoid":
        d_l = up * score * slope
    else:
        d_l = score * up - score * (score * up).sum(-1, keepdim=True)
    if s["dl"] is not None:
        d_l = d_l + s["dl"].double()
    return {"x": d_l.matmul(wg), "wg": d_l.t().matmul(x)}
