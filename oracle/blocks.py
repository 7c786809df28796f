"""Block operators in float64: the 8-bit linear layer, the gated feed-forward and
its gradients, query / key norm with rotation and its gradients, the residual's addition
with an RMS norm and its gradients, a linear layer with a low-rank adapter per row and
their gradients, the AdamW step.

The 8-bit scales are fp32 by definition; everything else is float64 throughout.
"""
import math

import numpy as np

F64 = np.float64


def quant_rows(x):
    """(q int8, scale float32): scale = max|x| / 127 rounded to fp32, at least 2^-126;
    q the nearest whole number to x / scale, ties to even; rows with a NaN or an
    infinity get scale NaN and zeros."""
    x = np.asarray(x, F64)
    ok = np.isfinite(x).all(1)
    xs = np.where(ok[:, None], x, 0.0)
    s = np.maximum((np.abs(xs).max(1) / 127.0).astype(np.float32), np.float32(2.0 ** -126))
    # (both are fp32 values: a quotient that is no tie differs from one by more than float64 loses)
    q = np.rint(xs / s.astype(F64)[:, None])
    return q.astype(np.int8), np.where(ok, s, np.float32(np.nan)).astype(np.float32)


def linear_i8(a, sa, w, sw, bias=None):
    acc = a.astype(np.int64) @ w.astype(np.int64).T
    y = acc.astype(F64) * np.asarray(sa, F64)[:, None] * np.asarray(sw, F64)[None]
    return y if bias is None else y + np.asarray(bias, F64)


def act(name, v):
    if name == "gelu":
        return 0.5 * v * (1 + np.tanh(math.sqrt(2 / math.pi) * (v + 0.044715 * v ** 3)))
    return v / (1 + np.exp(-v))


def act_grad(name, v):
    if name == "gelu":
        c = math.sqrt(2 / math.pi)
        t = np.tanh(c * (v + 0.044715 * v ** 3))
        return 0.5 * (1 + t) + 0.5 * v * (1 - t * t) * c * (1 + 3 * 0.044715 * v * v)
    s = 1 / (1 + np.exp(-v))
    return s + v * s * (1 - s)


def gated_pre(x, wg, wu, bg=None, bu=None):
    g, u = x @ wg.T, x @ wu.T
    return (g, u) if bg is None else (g + bg, u + bu)


def gated(name, g, u):
    return act(name, g) * u


def gated_grads(name, dout, x, wg, wu, g, u):
    """dict of dx, dwg, dwu, dbg, dbu, and the intermediate dg, du"""
    dg, du = dout * u * act_grad(name, g), dout * act(name, g)
    return dict(dg=dg, du=du, dx=dg @ wg + du @ wu, dwg=dg.T @ x, dwu=du.T @ x, dbg=dg.sum(0),
                dbu=du.sum(0))


def rotate(x, table, pos, pairing, inverse=False):
    """x [rows, heads, d]; table [n_pos, d/2, 2]; pos [rows], negative: not turned."""
    d = x.shape[-1]
    a, b = (x[..., 0::2], x[..., 1::2]) if pairing == "pairs" else (x[..., :d // 2], x[..., d // 2:])
    t = np.asarray(table, F64)[np.maximum(pos, 0)]
    still = (np.asarray(pos) < 0)[:, None]
    cos, sin = np.where(still, 1.0, t[..., 0])[:, None], np.where(still, 0.0, t[..., 1])[:, None]
    if inverse:
        sin = -sin
    y0, y1 = a * cos - b * sin, a * sin + b * cos
    return np.stack([y0, y1], -1).reshape(x.shape) if pairing == "pairs" else np.concatenate([y0, y1], -1)


def head_norm(x, w, eps):
    return x / np.sqrt((x * x).mean(-1, keepdims=True) + eps) * w


def qk_norm_rope(x, w, eps, table=None, pos=None, pairing="pairs"):
    n = head_norm(x, w, eps)
    return n if table is None else rotate(n, table, pos, pairing)


def qk_norm_rope_grads(dy, x, w, eps, table=None, pos=None, pairing="pairs"):
    """(dx, dw)"""
    dn = dy if table is None else rotate(dy, table, pos, pairing, inverse=True)
    r = 1 / np.sqrt((x * x).mean(-1, keepdims=True) + eps)
    n = x * r
    dw = (dn * n).sum((0, 1))
    dn = dn * w
    return r * (dn - n * (dn * n).mean(-1, keepdims=True)), dw


def add_rms_norm(h, w, eps):
    """y of the sum h [rows, K]"""
    return head_norm(h, 1.0 if w is None else w, eps)


def add_rms_norm_i8(h, w, eps):
    """(q int8, scale float64): t = h w, T = max|t|, scale = T / sqrt(mean h^2 + eps) / 127, q
    the nearest whole number to 127 t / T, ties to even.  h and w are fp32 values, so that the
    products fit float64 and 127 times them the 64 bits of a long double: exact."""
    t = np.asarray(h, F64) * (1.0 if w is None else np.asarray(w, F64))
    with np.errstate(over="ignore", invalid="ignore"):
        ok = np.isfinite(np.asarray(h, F64)).all(1) & np.isfinite(t.astype(np.float32)).all(1)
    ts = np.where(ok[:, None], t, 0.0)
    top = np.abs(ts).max(1, keepdims=True)
    L = np.longdouble
    assert np.finfo(L).nmant >= 63
    p, T = L(127) * np.abs(ts).astype(L), np.where(top > 0, top, 1.0).astype(L)
    n = np.rint(p / T)
    for side in (1, -1):
        edge = (n + L(side) / 2) * T
        over = (p > edge) | ((p == edge) & (n % 2 == 1)) if side > 0 else (p < edge) | ((p == edge) & (n % 2 == 1))
        n = np.where(over, n + side, n)
    q = np.where(top > 0, np.sign(ts) * n.astype(F64), 0.0).astype(np.int8)
    with np.errstate(divide="ignore", invalid="ignore"):
        s = top[:, 0] / np.sqrt((np.asarray(h, F64) ** 2).mean(1) + eps) / 127
    return q, np.where(ok, s, np.nan)


def add_rms_norm_grads(dy, h, w, dh, eps):
    """(gradient of the sum, dw)"""
    r = 1 / np.sqrt((h * h).mean(-1, keepdims=True) + eps)
    n = h * r
    d = dy * (1.0 if w is None else w)
    return (0.0 if dh is None else dh) + r * (d - n * (d * n).mean(-1, keepdims=True)), (dy * n).sum(0)


def adapter_rows(index, n, M):
    """For every adapter the rows that take it (index None: all rows adapter 0's)"""
    index = np.zeros(M, np.int64) if index is None else np.asarray(index)
    return [np.nonzero(index == i)[0] for i in range(n)]


def adapter_linear(x, w, a, b, bias=None, index=None, scale=None):
    """(y, t): y = x w^T + bias + t b_i^T, t = s_i x a_i^T, i the row's adapter (t 0 without one)"""
    y, t = x @ w.T, np.zeros((x.shape[0], a.shape[1]))
    if bias is not None:
        y = y + bias
    for i, rows in enumerate(adapter_rows(index, a.shape[0], x.shape[0])):
        t[rows] = (1.0 if scale is None else scale[i]) * x[rows] @ a[i].T
        y[rows] += t[rows] @ b[i].T
    return y, t


def adapter_linear_grads(dy, x, w, a, b, index=None, scale=None):
    """dict of dx, da, db, and u = s_i dy b_i"""
    _, t = adapter_linear(x, w, a, b, None, index, scale)
    dx, u = dy @ w, np.zeros_like(t)
    da, db = np.zeros_like(a), np.zeros_like(b)
    for i, rows in enumerate(adapter_rows(index, a.shape[0], x.shape[0])):
        u[rows] = (1.0 if scale is None else scale[i]) * dy[rows] @ b[i]
        dx[rows] += u[rows] @ a[i]
        da[i], db[i] = u[rows].T @ x[rows], dy[rows].T @ t[rows]
    return dict(dx=dx, da=da, db=db, u=u)


def adamw(p, g, m, v, step, lr, betas, eps, weight_decay, grad_scale=1.0):
    """(p, m, v) after one step"""
    b1, b2 = betas
    g = g * grad_scale
    m = b1 * m + (1 - b1) * g
    v = b2 * v + (1 - b2) * g * g
    way = m / (1 - b1 ** step) / (np.sqrt(v / (1 - b2 ** step)) + eps)
    return p - lr * (way + weight_decay * p), m, v
