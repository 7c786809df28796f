"""Block operators in float64: the 8-bit linear layer, the gated feed-forward and
its gradients, query / key norm with rotation and its gradients.

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
