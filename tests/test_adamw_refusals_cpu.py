"""What AdamW's Python class makes of gradients and weights that are not what they were, and its
formula against torch's (nothing here reaches a GPU)."""
import ctypes as C

import numpy as np
import pytest
import torch

import paper_2607_26566_amd as t2i
from oracle import blocks
from paper_2607_26566_amd import optim
from test_adamw_cpu import made
from test_block_ops_cpu import rng


def test_steps_are_those_of_torch():
    """torch takes lr weight_decay p off before the update by the moments, which do not depend on p:
    the same step, in float64 but for the roundings of a dozen operations (2^-53 each, of values up
    to 4) a step."""
    r = rng(3)
    p, g = r.normal(size=20), [r.normal(size=20) for _ in range(9)]
    t = torch.from_numpy(p.copy()).requires_grad_()
    opt = torch.optim.AdamW([t], lr=0.01, betas=(0.8, 0.95), eps=1e-6, weight_decay=0.1)
    q, m, v = p, np.zeros(20), np.zeros(20)
    for step, d in enumerate(g, 1):
        t.grad = torch.from_numpy(d)
        opt.step()
        q, m, v = blocks.adamw(q, d, m, v, step, 0.01, (0.8, 0.95), 1e-6, 0.1)
        assert np.abs(q - t.detach().numpy()).max() <= step * 12 * 2.0 ** -53 * 4


@pytest.fixture
def calls(monkeypatch):
    """addresses of the weights that reach the library, call by call"""
    seen = []

    class Lib:
        @staticmethod
        def t2i_op_adamw_step(dtype, kind, n, numel, p, *rest):
            seen.append(list((C.c_uint64 * n).from_address(p)))
            return 0
    monkeypatch.setattr(optim, "load", Lib)
    monkeypatch.setattr(optim, "_elsewhere", lambda *a: False)
    monkeypatch.setattr(optim, "_stream", lambda dev: 0)
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: False)
    return seen


def state():
    return dict(exp_avg=[made(4, 3), made(5)], exp_avg_sq=[made(4, 3), made(5)])


def test_gradients_that_are_no_tensors_are_refused(calls):
    opt = t2i.AdamW([made(4, 3), made(5)], step=2, **state())
    g = [made(4, 3), made(5)]
    for bad in ([g[0], None], [None, g[1]], [None, None], [g[0], 3.0], None, 7, made(2, 5), iter(g[:1]), iter([])):
        with pytest.raises(t2i.T2IError):
            opt.step(bad)
    assert opt.steps == 2 and not calls
    opt.step(t for t in g)
    opt.step(tuple(g))
    assert opt.steps == 4 and len(calls) == 2


def test_weights_put_into_the_list_are_the_ones_that_count(calls):
    kept = state()
    p = [made(4, 3), made(5)]
    opt = t2i.AdamW(p, step=2, **kept)
    g = [made(4, 3), made(5)]
    opt.step(g)
    new = made(5)
    opt.params[1] = new
    before = p[1]._version, new._version, p[0]._version, kept["exp_avg"][1]._version
    opt.step(g)
    assert calls[-1] == [p[0].data_ptr(), new.data_ptr()]
    assert (p[1]._version, new._version, p[0]._version, kept["exp_avg"][1]._version) == (
        before[0], before[1] + 1, before[2] + 1, before[3] + 1)
    # another tensor at the same place
    again = torch.nn.Parameter(new.data, requires_grad=False)
    opt.params[1] = again
    n = again._version
    opt.step(g)
    assert again._version == n + 1
    # what no step can take is refused, and the weights there were are taken again
    good, steps = opt.params[1], opt.steps
    for bad in (None, made(6), made(5, dtype=torch.bfloat16), torch.ones(5), kept["exp_avg"][1], p[0].view(-1)[:5],
                made(10)[::2], good[:3], good.view(1, 5), good.view(torch.int32)):
        opt.params[1] = bad
        with pytest.raises(t2i.T2IError):
            opt.step(g)
        with pytest.raises(t2i.T2IError):   # (not only the first time)
            opt.step(g)
    opt.params.pop()
    with pytest.raises(t2i.T2IError):
        opt.step(g)
    opt.params.append(good)
    assert opt.steps == steps
    opt.step(g)
    assert calls[-1] == [p[0].data_ptr(), good.data_ptr()]


def test_a_new_weight_that_requires_a_gradient_is_refused_as_the_first_ones_are(calls):
    opt = t2i.AdamW([made(4, 3), made(5)], step=2, **state())
    opt.params[0] = made(4, 3).requires_grad_()
    with pytest.raises(t2i.T2IError, match="no_grad"):
        opt.step([made(4, 3), made(5)])
    with torch.no_grad():
        opt.step([made(4, 3), made(5)])
    assert opt.steps == 3 and len(calls) == 1
