"""Plain fp64 forms of the products grouped by expert, the MXFP4 format and the
gradient clipping, written from their definitions (include/moe.h)."""
from __future__ import annotations

import numpy as np

MX_GRID = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def expert_rows(counts, n_rows):
    """[(first, n)] of the experts: a negative count is no row, and what lies
    behind n_rows is cut."""
    out, at = [], 0
    for c in counts:
        n = min(max(int(c), 0), n_rows - at)
        out.append((at, n))
        at += n
    return out


def grouped_product(x, w, counts, y0):
    """(y, bound): y[r] = w[e(r)] x[r] over a copy of y0, and the sums of the
    magnitudes of its terms (0 for rows without an expert)."""
    y, s = y0.copy(), np.zeros_like(y0)
    for e, (a, n) in enumerate(expert_rows(counts, x.shape[0])):
        y[a:a + n] = x[a:a + n] @ w[e].T
        s[a:a + n] = np.abs(x[a:a + n]) @ np.abs(w[e]).T
    return y, s


def grouped_product_backward(dy, x, w, counts, dx0, dw0):
    """(d_x, d_w, their sums of magnitudes) over copies of dx0 and dw0 (what d_w
    is added to)."""
    dx, dw = dx0.copy(), dw0.copy()
    sx, sw = np.zeros_like(dx0), np.abs(dw0)
    for e, (a, n) in enumerate(expert_rows(counts, dy.shape[0])):
        dx[a:a + n] = dy[a:a + n] @ w[e]
        sx[a:a + n] = np.abs(dy[a:a + n]) @ np.abs(w[e])
        dw[e] += dy[a:a + n].T @ x[a:a + n]
        sw[e] += np.abs(dy[a:a + n]).T @ np.abs(x[a:a + n])
    return dx, dw, sx, sw


def mx_quantize(v):
    """(codes uint8 [rows, cols / 2], scale bytes [rows, cols / 32]) of finite v."""
    rows, cols = v.shape
    b = np.asarray(v, np.float64).reshape(rows, cols // 32, 32)
    top = np.abs(b).max(-1)
    # frexp: top = m 2^x with m in [0.5, 1)
    e = np.where(top > 0, np.frexp(top)[1] - 3, -127)
    e = np.maximum(e, -127)
    a = np.abs(np.ldexp(b, -e[..., None]))
    code = np.zeros(a.shape, np.int64)
    off = a.copy()
    for k in range(1, 8):
        d = np.abs(a - MX_GRID[k])
        near = (d < off) | ((d == off) & (k % 2 == 0))
        code[near], off[near] = k, d[near]
    code += 8 * np.signbit(b)
    code = code.reshape(rows, cols // 2, 2)
    return (code[..., 0] + 16 * code[..., 1]).astype(np.uint8), (e + 127).astype(np.uint8)


def mx_values(codes, scales):
    """What codes and scales stand for (byte 255: NaN)."""
    k = np.stack((codes & 15, codes >> 4), -1).reshape(*codes.shape[:-1], -1, 32)
    v = MX_GRID[k & 7] * np.where(k & 8, -1.0, 1.0)
    p = np.ldexp(1.0, scales.astype(np.int64) - 127)
    p = np.where(scales == 255, np.nan, p)
    return (v * p[..., None]).reshape(*codes.shape[:-1], -1)


def clip(grads, max_norm):
    """(norm, scaled gradients); nothing is scaled where the norm is not finite."""
    norm = np.sqrt(sum(float((np.asarray(g, np.float64) ** 2).sum()) for g in grads))
    c = min(1.0, max_norm / (norm + 1e-6)) if np.isfinite(norm) else 1.0
    return norm, [np.asarray(g, np.float64) * c for g in grads]
