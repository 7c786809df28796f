"""AdamW on the host: the oracle against the step's meaning, and the refusals of the entry
point and of the Python class (nothing here reaches a GPU)."""
import ctypes as C

import numpy as np
import pytest
import torch

import paper_2607_26566_amd as t2i
from oracle import blocks
from test_block_ops_cpu import BF16, F32, INVALID, P, SHAPE, check_refusals, rng


def test_first_steps_by_hand():
    """The first step of zero moments goes by lr in the gradient's direction whatever its size; a
    constant gradient's does so for good; weights decay by lr weight_decay of themselves."""
    p, g = np.array([1.0, -2.0, 3.0]), np.array([1e-4, -50.0, 2.0])
    m = v = np.zeros(3)
    q = p
    for step in range(1, 6):
        q, m, v = blocks.adamw(q, g, m, v, step, 0.1, (0.9, 0.99), 0.0, 0.0)
        assert np.allclose(q, p - 0.1 * step * np.sign(g))
    q, _, _ = blocks.adamw(p, 0 * g, 0 * g, 0 * g, 1, 0.1, (0.9, 0.99), 1e-8, 0.5)
    assert np.allclose(q, p * 0.95)
    # a scale of the gradients is that of the gradients
    a = blocks.adamw(p, 3 * g, m, v, 6, 0.1, (0.9, 0.99), 1e-8, 0.1)
    b = blocks.adamw(p, g, m, v, 6, 0.1, (0.9, 0.99), 1e-8, 0.1, grad_scale=3.0)
    assert all(np.allclose(x, y) for x, y in zip(a, b))


def test_step_against_torch():
    r = rng(3)
    p, g = r.normal(size=20), [r.normal(size=20) for _ in range(4)]
    t = torch.from_numpy(p.copy()).requires_grad_()
    opt = torch.optim.AdamW([t], lr=0.01, betas=(0.8, 0.95), eps=1e-6, weight_decay=0.1)
    q, m, v = p, np.zeros(20), np.zeros(20)
    for step, d in enumerate(g, 1):
        t.grad = torch.from_numpy(d)
        opt.step()
        # (torch decays the weights first: the same to first order in lr, lr^2 weight_decay apart)
        q, m, v = blocks.adamw(q, d, m, v, step, 0.01, (0.8, 0.95), 1e-6, 0.1)
        assert np.allclose(q, t.detach().numpy(), atol=step * 2e-4 * 0.1)


def array(*v):
    return (C.c_void_p * len(v))(*v)


SPEC = dict(param_dtype=BF16, grad_dtype=BF16, n=2, numel=(C.c_int64 * 2)(8, 5), params=array(P, P), grads=array(P, P),
            exp_avg=array(P, P), exp_avg_sq=array(P, P), masters=array(P, P), lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8,
            weight_decay=0.1, step=1, lr_device=None, step_device=None, grad_scale=None, stream=None)


def test_adamw_step_refuses():
    nan = float("nan")
    check_refusals("t2i_op_adamw_step", SPEC, [
        (dict(param_dtype=2), INVALID), (dict(grad_dtype=-1), INVALID), (dict(n=0), SHAPE), (dict(numel=None), INVALID),
        (dict(params=None), INVALID), (dict(grads=None), INVALID), (dict(exp_avg=None), INVALID),
        (dict(exp_avg_sq=None), INVALID), (dict(masters=None), INVALID), (dict(param_dtype=F32), INVALID),
        (dict(beta1=1.0), INVALID), (dict(beta2=-0.1), INVALID), (dict(beta1=nan), INVALID), (dict(eps=-1.0), INVALID),
        (dict(eps=nan), INVALID), (dict(lr=nan), INVALID), (dict(weight_decay=float("inf")), INVALID),
        (dict(step=0), INVALID), (dict(lr_device=P + 2), INVALID), (dict(step_device=P + 1), INVALID),
        (dict(grad_scale=P + 3), INVALID), (dict(numel=(C.c_int64 * 2)(8, -1)), SHAPE),
        (dict(numel=(C.c_int64 * 2)(2 ** 33 + 1, 1)), SHAPE), (dict(params=array(P, None)), INVALID),
        (dict(grads=array(None, P)), INVALID), (dict(exp_avg=array(P, None)), INVALID),
        (dict(exp_avg_sq=array(None, P)), INVALID), (dict(masters=array(P, None)), INVALID),
        (dict(params=array(P, P + 1)), INVALID), (dict(grads=array(P + 1, P)), INVALID),
        (dict(exp_avg=array(P + 2, P)), INVALID), (dict(exp_avg_sq=array(P, P + 2)), INVALID),
        (dict(masters=array(P, P + 2)), INVALID)])


class OnDevice(torch.Tensor):
    """A host tensor that says it lies on device 0."""

    def get_device(self):
        return 0


def made(*shape, dtype=torch.float32):
    return torch.ones(shape, dtype=dtype).as_subclass(OnDevice)


def test_the_class_refuses():
    f, h = [made(4, 3), made(5)], [made(4, 3, dtype=torch.bfloat16), made(5, dtype=torch.bfloat16)]
    state = lambda: [made(4, 3), made(5)]  # noqa: E731
    for params, kw in (
            ([], {}), ([torch.ones(3)], {}), ([made(3, dtype=torch.float16)], {}), ([f[0], h[1]], {}),
            ([made(4, 3).T], {}), (f, dict(masters=state())), (f, dict(betas=(1.0, 0.9))), (f, dict(eps=-1.0)),
            (f, dict(lr=float("nan"))), (f, dict(weight_decay=float("inf"))), (f, dict(step=3)),
            (f, dict(exp_avg=state())), (f, dict(exp_avg=state(), exp_avg_sq=state()[:1])),
            (f, dict(exp_avg=state(), exp_avg_sq=[made(4, 3), made(6)])), (f, dict(exp_avg=state(), exp_avg_sq=h)),
            (f, dict(exp_avg=state(), exp_avg_sq=state(), step=-1)),
            (h, dict(masters=h, exp_avg=state(), exp_avg_sq=state())),
            ([f[0], f[0]], dict(exp_avg=[made(4, 3), made(4, 3)], exp_avg_sq=[made(4, 3), made(4, 3)])),
            (f, dict(exp_avg=f, exp_avg_sq=state())),
            (f, dict(exp_avg=[t.requires_grad_() for t in state()], exp_avg_sq=state()))):
        with pytest.raises(t2i.T2IError):
            t2i.AdamW(params, **kw)


def test_steps_refuse_and_mark_what_they_write(monkeypatch):
    from paper_2607_26566_amd import optim

    class Done:
        t2i_op_adamw_step = staticmethod(lambda *a: 0)
    monkeypatch.setattr(optim, "load", Done)
    monkeypatch.setattr(optim, "_elsewhere", lambda *a: False)
    monkeypatch.setattr(optim, "_stream", lambda dev: 0)
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: False)
    p, m, v = [made(4, 3), made(5)], [made(4, 3), made(5)], [made(4, 3), made(5)]
    opt = t2i.AdamW(p, exp_avg=m, exp_avg_sq=v, step=2)
    g = [made(4, 3), made(5)]
    before = [t._version for t in (*p, *m, *v)]
    opt.step(g)
    assert opt.steps == 3 and [t._version for t in (*p, *m, *v)] == [b + 1 for b in before]
    for bad in ([], g[:1], [g[0], made(6)], [g[0], made(5, dtype=torch.bfloat16)], [made(3, 4), g[1]],
                [made(3, 4).T, g[1]], [g[0], torch.ones(5)], [g[0], made(5, dtype=torch.float64)]):
        with pytest.raises(t2i.T2IError):
            opt.step(bad)
    for kw in (dict(lr=float("nan")), dict(lr=made(2)), dict(grad_scale=torch.ones(1)),
               dict(grad_scale=made(1, dtype=torch.bfloat16))):
        with pytest.raises(t2i.T2IError):
            opt.step(g, **kw)
    leaf = [g[0], made(5).requires_grad_()]
    with pytest.raises(t2i.T2IError, match="no_grad"):
        opt.step(leaf)
    with torch.no_grad():
        opt.step(leaf)
    p[0].requires_grad_()
    with pytest.raises(t2i.T2IError, match="no_grad"):
        opt.step(g)
    with torch.no_grad():
        opt.step(g)
    assert opt.steps == 5
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: True)
    with torch.no_grad(), pytest.raises(t2i.T2IError, match="capturable"):
        opt.step(g)
    assert opt.steps == 5
