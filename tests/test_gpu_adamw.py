"""The AdamW step on the GPU against its float64 definition (``oracle/blocks.py``), and the
operators of a fine-tuning step together.

Bounds count roundings (E = 2^-24): the moments' terms are off by up to 4 E (first) and 6 E
(second: all of one sign) of their sizes; the update by what the first moment is off by,
half of the second's with its factor's, square root's, sum's and quotient's own, 16 E; then
three more and the weight's own."""
import numpy as np
import pytest
import torch

import paper_2607_26566_amd as t2i
from oracle import blocks
from gpu_common import DEV, say, to_host
from test_gpu_block_ops import BF16, E, F32, NAME, U, dev, rnd, within

pytestmark = pytest.mark.gpu
A = np.abs
HYPER = dict(lr=0.02, betas=(0.9, 0.99), eps=1e-6, weight_decay=0.1)
# less than a lane's piece, a workgroup's elements and one more or less, several workgroups, none
SHAPES = [(1,), (7,), (8,), (3, 3), (2047,), (2048,), (2049,), (0,), (70, 1001), (5, 4, 3)]


def tensors(seed, shapes, std, dtype=F32, square=False):
    out = [rnd(seed + i, s, std, F32)[0] for i, s in enumerate(shapes)]
    return [(t.square() if square else t).to(dtype) for t in out]


def check_step(before, after, g, step, scale=1.0, hyper=HYPER):
    """before, after: (p, m, v) in float64"""
    p, m, v = before
    rp, rm, rv = blocks.adamw(p, g, m, v, step, hyper["lr"], hyper["betas"], hyper["eps"], hyper["weight_decay"], scale)
    b1, b2 = hyper["betas"]
    m_err = 4 * E * (A(b1 * m) + A((1 - b1) * g * scale))
    r1, denom = 1 / (1 - b1 ** step), np.sqrt(rv / (1 - b2 ** step)) + hyper["eps"]
    way = A(rm) * r1 / denom
    p_err = hyper["lr"] * (m_err * r1 / denom + 19 * E * way + 5 * E * hyper["weight_decay"] * A(p)) + E * A(rp)
    for got, ref, tol, what in ((after[0], rp, p_err, "p"), (after[1], rm, m_err, "m"), (after[2], rv, 6 * E * rv, "v")):
        within(got, ref, tol + 1e-44, what)


@pytest.mark.parametrize("dtype,gtype", [(F32, F32), (F32, BF16), (BF16, BF16), (BF16, F32)], ids=NAME.get)
def test_adamw_steps(dtype, gtype):
    say("adamw", NAME[dtype], NAME[gtype])
    p0 = tensors(1, SHAPES, 1.0)
    params = [p.to(dtype).contiguous() for p in p0]
    opt = t2i.AdamW(params, **HYPER)
    weights = params if dtype == F32 else opt.masters
    scale = torch.full((1,), 0.25, device=DEV)
    for step in range(1, 5):
        g = tensors(100 * step, SHAPES, 0.1, gtype)
        before = [[to_host(t) for t in ts] for ts in (weights, opt.exp_avg, opt.exp_avg_sq)]
        versions = [t._version for t in params]
        if step == 3:
            opt.step(g, grad_scale=scale, lr=0.5)
        elif step == 4:
            opt.step(g, lr=torch.tensor(0.125, device=DEV))
        else:
            opt.step(g)
        assert opt.steps == step and [t._version for t in params] == [x + 1 for x in versions]
        hyper = dict(HYPER, lr={3: 0.5, 4: 0.125}.get(step, HYPER["lr"]))
        for i, d in enumerate(g):
            check_step([b[i] for b in before], [to_host(ts[i]) for ts in (weights, opt.exp_avg, opt.exp_avg_sq)],
                       to_host(d), step, 0.25 if step == 3 else 1.0, hyper)
        if dtype == BF16:
            assert all(torch.equal(p, w.to(BF16)) for p, w in zip(params, weights))


@pytest.mark.parametrize("dtype", [F32, BF16], ids=NAME.get)
def test_many_tensors_take_the_steps_of_each(dtype):
    """150 tensors (three launches) against one at a time, some off 16 bytes and inside a larger
    buffer, whose other elements stay as they were."""
    r = np.random.default_rng(3)
    sizes = [int(n) for n in r.integers(1, 5000, 150)]

    def placed(seed, std, kind, square=False):
        flat = torch.full((sum(sizes) + 3 * 150 + 3,), 7.0, dtype=kind, device=DEV)
        out, at = [], 3
        for n, t in zip(sizes, tensors(seed, [(n,) for n in sizes], std, kind, square)):
            flat[at:at + n] = t
            out.append(flat[at:at + n])
            at += n + 3
        return out, flat
    low = dtype == BF16
    parts = dict(params=placed(1, 1.0, dtype), exp_avg=placed(200, 0.1, F32), exp_avg_sq=placed(400, 0.1, F32, True))
    if low:
        parts["masters"] = placed(600, 1.0, F32)
    g, gflat = placed(800, 0.1, dtype)
    one = {k: [t.clone() for t in v[0]] for k, v in parts.items()}
    opt = t2i.AdamW(**{k: v[0] for k, v in parts.items()}, step=6, **HYPER)
    opt.step(g)
    for i in range(150):
        t2i.AdamW(**{k: [v[i]] for k, v in one.items()}, step=6, **HYPER).step([g[i].clone()])
    inside = torch.ones(gflat.shape, dtype=torch.bool, device=DEV)
    at = 3
    for n in sizes:
        inside[at:at + n] = False
        at += n + 3
    for k, (ts, flat) in parts.items():
        assert all(torch.equal(a, b) for a, b in zip(ts, one[k])), k
        assert (flat[inside] == 7).all(), k


def test_adamw_values_that_are_not_finite_and_extremes():
    n = 40
    p, g = rnd(1, (n,), 1.0)[0], rnd(2, (n,), 1.0)[0]
    g[3], g[9], g[20], g[21] = float("nan"), float("inf"), 1e-30, 0.0
    opt = t2i.AdamW([p.clone()], **HYPER)
    opt.step([g])
    clean = g.clone()
    clean[[3, 9]] = 1.0
    ref = t2i.AdamW([p.clone()], **HYPER)
    ref.step([clean])
    keep = [i for i in range(n) if i not in (3, 9)]
    assert torch.equal(opt.params[0][keep], ref.params[0][keep]) and opt.params[0][[3, 9]].isnan().all()
    # betas of 0: moments are the gradient's; eps 0 and a zero gradient: 0 / 0, as the formula has it
    opt = t2i.AdamW([p.clone()], lr=0.1, betas=(0.0, 0.0), eps=0.0, weight_decay=0.0)
    opt.step([clean])
    assert torch.equal(opt.exp_avg[0], clean) and opt.params[0][21].isnan()
    within(opt.params[0][:20], to_host(p[:20]) - 0.1 * np.sign(to_host(clean[:20])), 8 * E * (1 + A(to_host(p[:20]))))


def test_adamw_captured_steps_count_on():
    shapes = [(300, 7), (2049,), (5,)]
    p = tensors(1, shapes, 1.0)
    eager = t2i.AdamW([t.clone() for t in p], **HYPER)
    graphed = t2i.AdamW([t.clone() for t in p], capturable=True, **HYPER)
    g, lr = tensors(50, shapes, 0.1), torch.tensor([0.02], device=DEV)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        graphed.step(g, lr=lr)
    torch.cuda.synchronize()
    eager.step(g, lr=lr)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        graphed.step(g, lr=lr)
    assert graphed.steps == 1
    for i in range(4):
        for t, s in zip(g, tensors(60 + 10 * i, shapes, 0.1)):
            t.copy_(s)
        lr.fill_(0.02 / (i + 1))
        graph.replay()
        torch.cuda.synchronize()
        eager.step(g, lr=lr)
        assert graphed.steps == eager.steps == i + 2
        for a, b in zip((*graphed.params, *graphed.exp_avg, *graphed.exp_avg_sq),
                        (*eager.params, *eager.exp_avg, *eager.exp_avg_sq)):
            # the device's powers of the betas: a last place of the factors
            assert np.allclose(to_host(a), to_host(b), rtol=4 * E, atol=8 * E)
    with pytest.raises(t2i.T2IError, match="capturable"):
        with torch.cuda.graph(torch.cuda.CUDAGraph()):
            eager.step(g)


@pytest.mark.parametrize("capturable", [False, True])
def test_adamw_refused_steps_do_not_count(capturable):
    say("refused step", capturable)
    (p,), (g,) = tensors(5, [(300,)], 1.0), tensors(6, [(300,)], 1.0)
    opt = t2i.AdamW([p.clone()], capturable=capturable, **HYPER)
    opt.eps = -1.0
    with pytest.raises(t2i.T2IError, match="eps"):
        opt.step([g])
    assert opt.steps == 0 and torch.equal(opt.params[0], p)
    opt.eps = HYPER["eps"]
    opt.step([g])
    assert opt.steps == 1
    zero = np.zeros(300)
    check_step((to_host(p), zero, zero), [to_host(t[0]) for t in (opt.params, opt.exp_avg, opt.exp_avg_sq)],
               to_host(g), 1)


def test_adamw_resumed_on_another_stream_and_exchanged_weights():
    shapes = [(30, 7), (2049,)]
    p, g = tensors(1, shapes, 1.0), tensors(50, shapes, 0.1)
    a = t2i.AdamW([t.clone() for t in p], **HYPER)
    a.step(g)
    b = t2i.AdamW([t.clone() for t in a.params], exp_avg=[t.clone() for t in a.exp_avg],
                  exp_avg_sq=[t.clone() for t in a.exp_avg_sq], step=a.steps, **HYPER)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    a.step(g)
    b.step(g, stream=side)
    side.synchronize()
    assert all(torch.equal(x, y) for x, y in zip((*a.params, *a.exp_avg, *a.exp_avg_sq),
                                                 (*b.params, *b.exp_avg, *b.exp_avg_sq)))
    # a weight whose storage was exchanged is the one that is updated
    old = b.params[0].clone()
    kept = b.params[0].data
    b.params[0].data = old.clone()
    a.step(g)
    b.step(g)
    assert torch.equal(kept, old) and all(torch.equal(x, y) for x, y in zip(a.params, b.params))


# ------------------------------------------------------------------ a fine-tuning step of the operators

class Norm(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, w, resid):
        y, h = t2i.add_rms_norm(x, w, resid)
        ctx.save_for_backward(h, w)
        return y, h

    @staticmethod
    def backward(ctx, dy, dh):
        h, w = ctx.saved_tensors
        dx, dresid, dw = t2i.add_rms_norm_backward(dy.contiguous(), h, w, dh.contiguous())
        return dx, dw, dx if dresid is None else dresid


class Adapted(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, w, a, b, index, scale):
        y, t = t2i.adapter_linear(x, w, a, b, index=index, scale=scale, save_t=True)
        ctx.save_for_backward(x, w, a, b, t, index, scale)
        return y

    @staticmethod
    def backward(ctx, dy):
        x, w, a, b, t, index, scale = ctx.saved_tensors
        dx, da, db = t2i.adapter_linear_backward(dy.contiguous(), x, w, a, b, t, index=index, scale=scale)
        return dx, None, da, db, None, None


def fine_tuning(dtype):
    M, K, N, n, r = 70, 136, 136, 3, 8
    o = dict(x=rnd(1, (M, K), 1.0, dtype)[0], resid=rnd(2, (M, K), 1.0, F32)[0], w=rnd(3, (N, K), K ** -0.5, dtype)[0],
             norm=rnd(4, (K,), 0.1, dtype)[0] + 1, a=rnd(5, (n, r, K), K ** -0.5, dtype)[0],
             b=rnd(6, (n, N, r), r ** -0.5, dtype)[0], dy=rnd(7, (M, N), 1.0, dtype)[0], dh=rnd(8, (M, K), 1.0, F32)[0])
    index = torch.from_numpy(np.random.default_rng(9).integers(-1, n, M).astype(np.int32)).to(DEV)
    return o, index, torch.tensor([0.5, 1.0, 2.0], device=DEV)


def test_a_fine_tuning_step_of_the_operators_together():
    """A residual block's norm and adapted layer under automatic differentiation, then AdamW on the
    adapters and the norm's weight, against float64: gradients first, then the step's weights."""
    for dtype in (F32, BF16):
        o, index, scale = fine_tuning(dtype)
        leaves = {k: o[k].clone().requires_grad_() for k in ("x", "resid", "norm", "a", "b")}
        y, h = Norm.apply(leaves["x"], leaves["norm"], leaves["resid"])
        z = Adapted.apply(y, o["w"], leaves["a"], leaves["b"], index, scale)
        torch.autograd.backward([z, h], [o["dy"], o["dh"]])
        r = {k: to_host(v) for k, v in o.items()}
        hh = to_host((o["resid"] + o["x"].float()))
        yy = blocks.add_rms_norm(hh, r["norm"], 1e-6)
        ix = index.cpu().numpy()
        ref = blocks.adapter_linear_grads(r["dy"], yy, r["w"], r["a"], r["b"], ix, to_host(scale))
        ds, dn = blocks.add_rms_norm_grads(ref["dx"], hh, r["norm"], r["dh"], 1e-6)
        for got, want in ((leaves["x"].grad, ds), (leaves["resid"].grad, ds), (leaves["norm"].grad, dn),
                          (leaves["a"].grad, ref["da"]), (leaves["b"].grad, ref["db"])):
            # y, t, u, dx and the result are rounded, one after the other, to the type
            rel = np.linalg.norm(to_host(got) - want) / np.linalg.norm(want)
            assert rel < 5 * U[dtype] + 300 * E, rel
        names = ("norm", "a", "b")
        opt = t2i.AdamW([leaves[k].detach() for k in names], lr=0.1, weight_decay=0.1)
        before = [to_host(leaves[k]) for k in names]
        grads = [leaves[k].grad for k in names]
        opt.step(grads)
        for k, b, g in zip(names, before, grads):
            p, _, _ = blocks.adamw(b, to_host(g), 0 * b, 0 * b, 1, 0.1, (0.9, 0.999), 1e-8, 0.1)
            tol = 40 * E * (0.1 + A(p)) + (U[dtype] * A(p) if dtype == BF16 else 0)
            within(leaves[k], p, tol, k)


def test_an_8_bit_layer_behind_the_norm():
    """add_rms_norm_i8's codes through linear_i8, beside the layer of the unrounded norm."""
    x, w, resid = rnd(1, (300, 520), 1.0, BF16)[0], rnd(2, (520,), 0.1, BF16)[0] + 1, rnd(3, (300, 520), 1.0, F32)[0]
    q, s, h = t2i.add_rms_norm_i8(x, w, resid)
    wq, ws = t2i.quant_rows(rnd(4, (264, 520), 0.05, BF16)[0])
    out = t2i.linear_i8(q, s, wq, ws, K=520, dtype=F32)
    codes, scales = blocks.add_rms_norm_i8(to_host(h), to_host(w), 1e-6)
    ref = blocks.linear_i8(codes, scales, wq.cpu().numpy()[:, :520], to_host(ws))
    # the scale's 42 E, and the layer's four roundings
    within(out, ref, 46 * E * A(ref))


def test_a_whole_step_in_a_graph():
    """Norm, adapted layer, their gradients and AdamW captured together, replayed against eager calls."""
    o, index, scale = fine_tuning(BF16)

    def build():
        w = [o["norm"].clone(), o["a"].clone(), o["b"].clone()]
        opt = t2i.AdamW(w, lr=0.05, capturable=True)

        def work():
            y, h = t2i.add_rms_norm(o["x"], w[0], o["resid"])
            z, t = t2i.adapter_linear(y, o["w"], w[1], w[2], index=index, scale=scale, save_t=True)
            dx, da, db = t2i.adapter_linear_backward(o["dy"], y, o["w"], w[1], w[2], t, index=index, scale=scale)
            ds, _, dn = t2i.add_rms_norm_backward(dx, h, w[0], o["dh"])
            opt.step([dn, da, db])
            return z, ds
        return opt, work
    opt, work = build()
    ref, again = build()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        work()
    torch.cuda.synchronize()
    again()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = work()
    for _ in range(4):
        graph.replay()
        torch.cuda.synchronize()
        want = again()
        for a, b in zip((*out, *opt.masters, *opt.params, *opt.exp_avg, *opt.exp_avg_sq),
                        (*want, *ref.masters, *ref.params, *ref.exp_avg, *ref.exp_avg_sq)):
            assert torch.equal(a, b)
