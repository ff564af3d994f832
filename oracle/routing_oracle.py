"""CPU oracle of the routing rules and the layer norm in float64, written from
their definitions (include/moe.h), token by token.

Inputs are numpy arrays of any float type, taken as the exact values they
hold.  Nothing here uses the library under test.
"""
from __future__ import annotations

import numpy as np

SOFTMAX, SIGMOID = 0, 1


class Rule:
    """What moe_router_desc says, without sizes and types."""

    def __init__(self, top_k, score=SOFTMAX, n_groups=1, top_groups=1, group_best=1,
                 renormalize=True, scale=1.0):
        self.top_k, self.score, self.n_groups = top_k, score, n_groups
        self.top_groups, self.group_best = top_groups, group_best
        self.renormalize, self.scale = renormalize, float(np.float32(scale))


def _sigmoid(l):
    return np.where(l >= 0, 1.0 / (1.0 + np.exp(-np.abs(l))),
                    np.exp(-np.abs(l)) / (1.0 + np.exp(-np.abs(l))))


def scores(rule, l):
    """Scores of one token's logits; a logit that is not finite scores 0."""
    fin = np.isfinite(l)
    s = np.zeros(l.shape)
    if rule.score == SIGMOID:
        s[fin] = _sigmoid(l[fin])
    elif fin.any():
        e = np.exp(l[fin] - l[fin].max())
        s[fin] = e / e.sum()
    return s


def select(rule, l, bias=None):
    """Selected experts of one token, slot 0 first; -1 where none is left."""
    E, G = l.shape[0], rule.n_groups
    fit = np.isfinite(l)
    s = scores(rule, l)
    key = l.copy()
    if bias is not None:
        fit &= np.isfinite(bias)
        key = s + np.where(np.isfinite(bias), bias, 0.0)
    if G > 1:
        size = E // G
        total = []
        for g in range(G):
            of = [(key if bias is not None else s)[e] for e in range(g * size, (g + 1) * size) if fit[e]]
            of = sorted(of, reverse=True)[:rule.group_best]
            total.append(sum(of) if of else -np.inf)
        order = sorted(range(G), key=lambda g: (-total[g], g))[:rule.top_groups]
        for g in range(G):
            if g not in order:
                fit[g * size:(g + 1) * size] = False
    order = sorted((e for e in range(E) if fit[e]), key=lambda e: (-key[e], e))[:rule.top_k]
    return np.array(order + [-1] * (rule.top_k - len(order)), dtype=np.int32)


def shares(rule, l, idx):
    """Selected scores over their sum (0 in slots without an expert), formed
    from logarithms so that scores that underflow keep their ratios."""
    out = np.zeros(len(idx))
    on = idx >= 0
    if on.any():
        v = l[idx[on]]
        v = np.minimum(v, 0.0) - np.log1p(np.exp(-np.abs(v))) if rule.score == SIGMOID else v
        e = np.exp(v - v.max())
        out[on] = e / e.sum()
    return out


def weights(rule, l, idx):
    if rule.renormalize:
        return rule.scale * shares(rule, l, idx)
    return rule.scale * np.where(idx >= 0, scores(rule, l)[np.maximum(idx, 0)], 0.0)


def route(rule, x, wg, bias=None):
    """(idx [T, K], w [T, K], logits [T, E], count [E])."""
    with np.errstate(invalid="ignore", over="ignore"):
        l = np.asarray(x, np.float64) @ np.asarray(wg, np.float64).T
    b = None if bias is None else np.asarray(bias, np.float64)
    idx = np.stack([select(rule, r, b) for r in l])
    w = np.stack([weights(rule, r, i) for r, i in zip(l, idx)])
    return idx, w, l, np.bincount(idx[idx >= 0], minlength=wg.shape[0]).astype(np.int32)


def logit_gradient(rule, l, idx, dw, dl=None):
    """Gradient of one token's logits: of sum(w * dw) + sum(logits * dl)."""
    g = np.zeros(l.shape)
    on = (idx >= 0) & (idx < len(l))
    on &= np.isfinite(l[np.where(on, idx, 0)])
    ids, up = idx[on], rule.scale * np.asarray(dw, np.float64)[on]
    s = scores(rule, l)
    if rule.renormalize:
        p = shares(rule, l, ids)
        slot = p * (up - (up * p).sum())
        if rule.score == SIGMOID:
            slot = slot * _sigmoid(-l[ids])
        np.add.at(g, ids, slot)
    elif rule.score == SIGMOID:
        np.add.at(g, ids, up * s[ids] * _sigmoid(-l[ids]))
    else:
        np.add.at(g, ids, up * s[ids])
        g -= s * (up * s[ids]).sum()
    return g if dl is None else g + np.asarray(dl, np.float64)


def route_backward(rule, x, wg, logits, idx, dw, dl=None):
    """(d_x [T, d], d_wg [E, d], gradient of the logits [T, E])."""
    g = np.stack([logit_gradient(rule, np.asarray(logits[t], np.float64), idx[t], dw[t],
                                 None if dl is None else dl[t]) for t in range(len(idx))])
    return g @ np.asarray(wg, np.float64), g.T @ np.asarray(x, np.float64), g


def eq2_precisions(share, idx, tags, t1, t2):
    """Precisions (0 high, 1 low, 2 skipped) of one token's slots: slots ranked
    by share, ties to the lower slot; see the Eq. 2 rule of the layer."""
    order = sorted(range(len(idx)), key=lambda k: (-share[k], k))
    prec, above = np.full(len(idx), 2, np.int8), 0.0
    for n, k in enumerate(order):
        if idx[k] < 0:
            continue
        tag = int(tags[idx[k]])
        if tag in (0, 5):
            prec[k] = 0
        elif tag in (1, 2):
            prec[k] = 1
        else:
            prec[k] = 0 if n == 0 or above <= t1 else 1 if above <= t2 else 2
        above += share[k]
    return prec


def layernorm(h, gain=None, bias=None, eps=1e-5):
    h = np.asarray(h, np.float64)
    c = h - h.mean(-1, keepdims=True)
    n = c / np.sqrt((c * c).mean(-1, keepdims=True) + eps)
    x = n if gain is None else n * np.asarray(gain, np.float64)
    return x if bias is None else x + np.asarray(bias, np.float64)


def layernorm_backward(dx, h, gain=None, eps=1e-5):
    """(d_h, d_gain, d_bias)."""
    dx, h = np.asarray(dx, np.float64), np.asarray(h, np.float64)
    c = h - h.mean(-1, keepdims=True)
    r = 1.0 / np.sqrt((c * c).mean(-1, keepdims=True) + eps)
    n = c * r
    a = dx if gain is None else dx * np.asarray(gain, np.float64)
    dh = r * (a - a.mean(-1, keepdims=True) - n * (a * n).mean(-1, keepdims=True))
    return dh, (dx * n).sum(0), dx.sum(0)
