"""The residual's addition with an RMS norm on the host: the oracle's formulas against
differences and whole-number arithmetic, and the refusals of the entry points (nothing
here reaches a GPU: each call fails its argument checks)."""
from fractions import Fraction

import numpy as np
import pytest
import torch

import paper_2607_26566_amd as t2i
from paper_2607_26566_amd import _lib
from oracle import blocks
from test_block_ops_cpu import BF16, F32, INVALID, P, SHAPE, WORKSPACE, OnDevice, check_refusals, rng


@pytest.mark.parametrize("weight", [True, False])
def test_gradients_against_differences(weight):
    r = rng(4)
    rows, K, eps = 3, 7, 1e-3
    resid, x, dy, dz = (r.normal(size=(rows, K)) for _ in range(4))
    w = r.normal(size=K) if weight else None

    # (the sum goes on by itself, too: dz)
    def loss(a, b, c):
        h = a + b
        return (blocks.add_rms_norm(h, c, eps) * dy + h * dz).sum()
    ds, dw = blocks.add_rms_norm_grads(dy, resid + x, w, dz, eps)
    for v, got, f in ((x, ds, lambda t: loss(resid, t, w)), (resid, ds, lambda t: loss(t, x, w)),
                      (w, dw, lambda t: loss(resid, x, t))):
        if v is None:
            continue
        num = np.zeros_like(v)
        for i in np.ndindex(*v.shape):
            hi, lo = v.copy(), v.copy()
            hi[i] += 1e-6
            lo[i] -= 1e-6
            num[i] = (f(hi) - f(lo)) / 2e-6
        # central differences: h^2 f''' / 6 + 2^-53 |f| / h, both below 1e-8 here
        assert np.allclose(got, num, rtol=1e-6, atol=1e-7)


def test_codes_by_whole_number_arithmetic():
    r = rng(6)
    h = np.concatenate([r.normal(size=(20, 30)), np.arange(600).reshape(20, 30) / 2]).astype(np.float32)
    w = r.normal(size=30).astype(np.float32)
    for weight in (None, w, np.float32(2.0) ** r.integers(-3, 3, 30)):
        q, s = blocks.add_rms_norm_i8(h, weight, 0.0)
        for row, codes, sc in zip(h, q, s):
            t = [Fraction(float(a)) * Fraction(float(b)) for a, b in zip(row, np.ones(30) if weight is None else weight)]
            top = max(map(abs, t))
            for v, n in zip(t, codes):
                f = 127 * v / top
                assert abs(f - int(n)) < Fraction(1, 2) or (abs(f - int(n)) == Fraction(1, 2) and n % 2 == 0)
            norm = np.array([float(v) for v in t]) / np.sqrt((row.astype(np.float64) ** 2).mean())
            assert np.abs(codes * sc - norm).max() <= sc * (0.5 + 1e-9)
    q, s = blocks.add_rms_norm_i8(np.array([[0.0, 0], [np.nan, 1], [1, np.inf], [1, 1e30]]), np.float32([1, 1e10]), 1.0)
    assert s[0] == 0 and np.isnan(s[1:]).all() and not q.any()


NORM = dict(dtype=BF16, resid_dtype=F32, rows=3, K=130, x=P, ldx=130, resid=P, ldr=130, w=P, eps=1e-6, h=P, ldh=130,
            y=P, ldy=130, stream=None)
REFUSED = [
    (dict(dtype=2), INVALID), (dict(resid_dtype=2), INVALID), (dict(dtype=F32, resid_dtype=BF16), INVALID),
    (dict(resid=None), INVALID), (dict(rows=0), SHAPE), (dict(rows=-1), SHAPE), (dict(K=0), SHAPE),
    (dict(rows=2 ** 26 - 4), SHAPE), (dict(K=2 ** 20 + 1, ldx=2 ** 21, ldr=2 ** 21, ldh=2 ** 21, ldy=2 ** 21), SHAPE),
    (dict(rows=2 ** 22, K=2049, ldx=2049, ldr=2049, ldh=2049, ldy=2049), SHAPE),
    (dict(x=None), INVALID), (dict(h=None), INVALID), (dict(y=None), INVALID), (dict(ldx=129), SHAPE),
    (dict(ldr=129), SHAPE), (dict(ldh=129), SHAPE), (dict(x=P + 1), INVALID), (dict(w=P + 1), INVALID),
    (dict(resid=P + 2), INVALID), (dict(h=P + 2), INVALID), (dict(eps=-1.0), INVALID),
    (dict(eps=float("nan")), INVALID), (dict(eps=float("inf")), INVALID)]


def test_add_rms_norm_refuses():
    check_refusals("t2i_op_add_rms_norm", NORM, REFUSED + [(dict(ldy=129), SHAPE), (dict(y=P + 1), INVALID)])


def test_add_rms_norm_i8_refuses():
    spec = {k: v for k, v in NORM.items() if k not in ("y", "ldy", "stream")}
    spec.update(q=P, ldq=256, scale=P, stream=None)
    drop = [({k: v for k, v in c.items() if k != "ldy"}, s) for c, s in REFUSED if "y" not in c]
    check_refusals("t2i_op_add_rms_norm_i8", spec, drop + [
        (dict(q=None), INVALID), (dict(scale=None), INVALID), (dict(ldq=240), SHAPE), (dict(ldq=264), SHAPE),
        (dict(q=P + 8), INVALID), (dict(scale=P + 2), INVALID)])


def test_add_rms_norm_backward_refuses():
    lib = t2i.load()
    n = lib.t2i_op_add_rms_norm_backward_ws_bytes(30, 130)
    assert n > 0 and n % 4 == 0 and lib.t2i_op_add_rms_norm_backward_ws_bytes(16, 130) == 0
    for rows, K in ((0, 5), (5, 0), (5, 2 ** 20 + 1), (2 ** 26, 5)):
        assert lib.t2i_op_add_rms_norm_backward_ws_bytes(rows, K) == 0
    spec = dict(dtype=BF16, resid_dtype=F32, rows=30, K=130, dy=P, lddy=130, h=P, ldh=130, w=P, eps=1e-6, dh=P,
                lddh=130, dx=P, lddx=130, dresid=P, lddr=130, dw=P, ws=P, ws_bytes=n, stream=None)
    check_refusals("t2i_op_add_rms_norm_backward", spec, [
        (dict(dtype=2), INVALID), (dict(resid_dtype=-1), INVALID), (dict(dtype=F32, resid_dtype=BF16), INVALID),
        (dict(rows=0), SHAPE), (dict(K=0), SHAPE), (dict(dy=None), INVALID), (dict(h=None), INVALID),
        (dict(dx=None), INVALID), (dict(lddy=129), SHAPE), (dict(ldh=129), SHAPE), (dict(lddx=129), SHAPE),
        (dict(lddh=129), SHAPE), (dict(lddr=129), SHAPE), (dict(dy=P + 1), INVALID), (dict(h=P + 2), INVALID),
        (dict(dh=P + 2), INVALID), (dict(dx=P + 1), INVALID), (dict(dresid=P + 2), INVALID), (dict(w=P + 1), INVALID),
        (dict(dw=P + 1), INVALID), (dict(ws=P + 4), INVALID), (dict(ws=None), WORKSPACE),
        (dict(ws_bytes=n - 1), WORKSPACE), (dict(eps=-1e-9), INVALID)])


def test_python_calls_refuse_what_differentiation_follows(monkeypatch):
    from paper_2607_26566_amd import ops

    class Through(Exception):
        pass

    def through(*a):
        raise Through
    monkeypatch.setattr(ops, "_elsewhere", through)
    mk = lambda *s: torch.ones(s).as_subclass(OnDevice)  # noqa: E731
    for call, operands in ((t2i.add_rms_norm, [mk(4, 64), mk(64), mk(4, 64)]),
                           (t2i.add_rms_norm_i8, [mk(4, 64), mk(64), mk(4, 64)]),
                           (t2i.add_rms_norm_backward, [mk(4, 64), mk(4, 64), mk(64), mk(4, 64)])):
        with pytest.raises(Through):
            call(*operands)
        for i, t in enumerate(operands):
            args = [*operands[:i], t.clone().requires_grad_(), *operands[i + 1:]]
            with pytest.raises(t2i.T2IError, match="requires a gradient"):
                call(*args)
            with torch.no_grad(), pytest.raises(Through):
                call(*args)
