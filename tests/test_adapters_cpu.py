"""Adapters of many requests on the host: the oracle's formulas against differences and
against the merged weights, and the refusals of the entry points (nothing here reaches a
GPU: each call fails its argument checks)."""
import numpy as np
import pytest
import torch

import paper_2607_26566_amd as t2i
from paper_2607_26566_amd import _lib
from oracle import blocks
from test_block_ops_cpu import BF16, F32, INVALID, P, SHAPE, WORKSPACE, OnDevice, check_refusals, rng


def operands(r, M, N, K, n, rank):
    return dict(x=r.normal(size=(M, K)), w=r.normal(size=(N, K)), a=r.normal(size=(n, rank, K)),
                b=r.normal(size=(n, N, rank)), scale=r.uniform(0.5, 2, n))


def test_rows_are_those_of_merged_weights():
    r = rng(1)
    p = operands(r, 7, 5, 6, 3, 2)
    index, bias = np.array([2, -1, 0, 2, 3, 1, 0]), r.normal(size=5)
    y, t = blocks.adapter_linear(**p, bias=bias, index=index)
    for m, i in enumerate(index):
        own = p["w"] + (p["scale"][i] * p["b"][i] @ p["a"][i] if 0 <= i < 3 else 0)
        assert np.allclose(y[m], own @ p["x"][m] + bias)
    assert not t[1].any() and not t[4].any()


@pytest.mark.parametrize("index", [None, [1, -1, 0, 1, 5]])
def test_gradients_against_differences(index):
    r = rng(2)
    p = operands(r, 5, 4, 3, 3 if index else 1, 2)
    dy = r.normal(size=(5, 4))
    scale = p.pop("scale")
    loss = lambda q: (blocks.adapter_linear(**q, index=index, scale=scale)[0] * dy).sum()  # noqa: E731
    got = blocks.adapter_linear_grads(dy, **p, index=index, scale=scale)
    for name in ("x", "a", "b"):
        num = np.zeros_like(p[name])
        for i in np.ndindex(*p[name].shape):
            hi, lo = ({**p, name: p[name].copy()} for _ in range(2))
            hi[name][i] += 1e-6
            lo[name][i] -= 1e-6
            num[i] = (loss(hi) - loss(lo)) / 2e-6
        # central differences: the loss is of second degree in a (in b) at most, 2^-53 |f| / h below 1e-8
        assert np.allclose(got["d" + name], num, rtol=1e-6, atol=1e-7), name


FWD = dict(dtype=BF16, epilogue=0, M=3, N=16, K=136, x=P, ldx=136, w=P, ldw=136, bias=P, n=2, rank=5, a=P, b=P,
           scale=P, index=P, t=P, ldt=32, out=P, ldo=16, resid=None, ldr=16, resid_copy=None, gate=None, stream=None)
COMMON = [
    (dict(dtype=2), INVALID), (dict(M=0), SHAPE), (dict(N=0), SHAPE), (dict(K=0), SHAPE), (dict(n=0), SHAPE),
    (dict(rank=0), SHAPE), (dict(rank=129, ldt=160), SHAPE), (dict(n=32768), SHAPE), (dict(M=2 ** 24 + 1), SHAPE),
    (dict(M=2 ** 20, N=2 ** 20), SHAPE), (dict(n=32767, rank=128, K=4096, ldx=4096, ldw=4096), SHAPE),
    (dict(x=None), INVALID), (dict(w=None), INVALID), (dict(a=None), INVALID), (dict(b=None), INVALID),
    (dict(t=None), INVALID), (dict(ldx=128), SHAPE), (dict(ldw=135), SHAPE), (dict(ldx=140), SHAPE),
    (dict(ldw=140), SHAPE), (dict(K=132), SHAPE), (dict(N=12), SHAPE), (dict(ldt=24), SHAPE), (dict(ldt=36), SHAPE),
    (dict(rank=33), SHAPE), (dict(ldx=2 ** 22), SHAPE), (dict(ldw=2 ** 22), SHAPE), (dict(x=P + 8), INVALID),
    (dict(w=P + 8), INVALID), (dict(a=P + 8), INVALID), (dict(b=P + 1), INVALID), (dict(scale=P + 2), INVALID),
    (dict(index=P + 2), INVALID), (dict(t=P + 8), INVALID), (dict(dtype=F32, x=P + 2), INVALID)]


def test_adapter_linear_refuses():
    res = dict(epilogue=_lib.T2I_EPI_RESID, out=None, resid=P)
    gated = dict(res, epilogue=_lib.T2I_EPI_RESID_GATED, gate=P)
    check_refusals("t2i_op_adapter_linear", FWD, COMMON + [
        (dict(epilogue=5), INVALID), (dict(epilogue=-1), INVALID), (dict(out=None), INVALID), (dict(ldo=15), INVALID),
        (dict(out=P + 1), INVALID), (dict(bias=P + 1), INVALID), (dict(res, resid=None), INVALID),
        (dict(res, ldr=15), INVALID), (dict(res, resid=P + 2), INVALID), (dict(res, resid_copy=P + 1), INVALID),
        (dict(gated, gate=None), INVALID), (dict(gated, gate=P + 2), INVALID)])


def test_adapter_linear_backward_refuses():
    lib = t2i.load()
    size = lib.t2i_op_adapter_linear_backward_ws_bytes
    need = size(BF16, 3, 16, 136, 2, 5)
    assert need > 0 and need % 256 == 0
    for bad in ((2, 3, 16, 136, 2, 5), (BF16, 0, 16, 136, 2, 5), (BF16, 3, 16, 136, 2, 129), (BF16, 3, 16, 136, 0, 5)):
        assert size(*bad) == 0
    spec = dict(dtype=BF16, M=3, N=16, K=136, dy=P, lddy=16, x=P, ldx=136, w=P, ldw=136, n=2, rank=5, a=P, b=P,
                scale=P, index=P, t=P, ldt=32, dx=P, lddx=136, da=P, db=P, ws=P, ws_bytes=need, stream=None)
    check_refusals("t2i_op_adapter_linear_backward", spec, COMMON + [
        (dict(dy=None), INVALID), (dict(ws=None), INVALID), (dict(dx=None, da=None, db=None), INVALID),
        (dict(lddy=8), SHAPE), (dict(lddx=128), SHAPE), (dict(lddy=20), SHAPE), (dict(lddx=140), SHAPE),
        (dict(lddy=2 ** 22), SHAPE), (dict(dy=P + 8), INVALID), (dict(dx=P + 8), INVALID), (dict(da=P + 1), INVALID),
        (dict(db=P + 1), INVALID), (dict(ws=P + 128), INVALID), (dict(ws_bytes=need - 1), WORKSPACE),
        # more slices of the sums than a launch holds
        (dict(dtype=F32, n=32767, M=2 ** 16, K=2 ** 14, N=2 ** 14, ldx=2 ** 14, ldw=2 ** 14, lddy=2 ** 14, lddx=2 ** 14,
              rank=8), SHAPE)])
    assert b"launch" in lib.t2i_ops_last_error()


def test_python_calls_refuse_what_differentiation_follows(monkeypatch):
    from paper_2607_26566_amd import ops

    class Through(Exception):
        pass

    def through(*a):
        raise Through
    monkeypatch.setattr(ops, "_elsewhere", through)
    mk = lambda *s: torch.ones(s).as_subclass(OnDevice)  # noqa: E731
    index = torch.zeros(4, dtype=torch.int32).as_subclass(OnDevice)
    for call, operands in (
            (lambda x, w, a, b, c, s, r, g: t2i.adapter_linear(x, w, a, b, c, index=index, scale=s, epilogue="resid_gated",
                                                               resid=r, gate=g),
             [mk(4, 64), mk(8, 64), mk(2, 3, 64), mk(2, 8, 3), mk(8), mk(2), mk(4, 8), mk(8)]),
            (lambda dy, x, w, a, b, t, s: t2i.adapter_linear_backward(dy, x, w, a, b, t, index=index, scale=s),
             [mk(4, 8), mk(4, 64), mk(8, 64), mk(2, 3, 64), mk(2, 8, 3), mk(4, 32), mk(2)])):
        with pytest.raises(Through):
            call(*operands)
        for i, t in enumerate(operands):
            args = [*operands[:i], t.clone().requires_grad_(), *operands[i + 1:]]
            with pytest.raises(t2i.T2IError, match="requires a gradient"):
                call(*args)
            with torch.no_grad(), pytest.raises(Through):
                call(*args)
