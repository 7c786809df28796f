"""The block operators on the GPU against their float64 definitions (``oracle/blocks.py``).

Bounds count roundings.  U is half a step of the result's type relative to the
value (bf16 2^-8, fp32 2^-24); E = 2^-24.  A sum of n products in fp32 is off by
at most n E times the sum of the products' sizes; the activations' hardware
exponential and reciprocal are within a few E of a value of their argument's
size, taken as 2^-20."""
import ctypes as C

import numpy as np
import pytest
import torch

import paper_2607_26566_amd as t2i
from paper_2607_26566_amd import _lib
from oracle import blocks, dit
from gpu_common import DEV, rel_l2, say, to_host

pytestmark = pytest.mark.gpu

E = 2.0 ** -24
BF16, F32 = torch.bfloat16, torch.float32
U = {BF16: 2.0 ** -8, F32: E}
NAME = {BF16: "bf16", F32: "f32"}
DTYPES = pytest.mark.parametrize("dtype", [BF16, F32], ids=NAME.get)


def dev(a, dtype=F32):
    return torch.from_numpy(np.ascontiguousarray(a)).to(DEV).to(dtype)


def rnd(seed, shape, std=1.0, dtype=F32):
    """(device tensor, the same values in float64)"""
    t = dev(np.random.default_rng(seed).standard_normal(shape, dtype=np.float32) * np.float32(std), dtype)
    return t, to_host(t)


def within(got, ref, tol, what=""):
    got = to_host(got) if torch.is_tensor(got) else got
    assert got.shape == ref.shape
    assert np.isfinite(got).all(), what
    bad = np.abs(got - ref) - tol
    assert (bad <= 0).all(), (what, float(bad.max()), np.unravel_index(bad.argmax(), bad.shape))


def padded(t, extra, fill=7.0):
    """(a copy of matrix t whose rows are `extra` elements further apart, its buffer)"""
    buf = torch.full((t.shape[0] + 1, t.shape[1] + extra), fill, dtype=t.dtype, device=DEV)
    buf[:-1, :t.shape[1]] = t
    return buf[:-1, :t.shape[1]], buf


# ------------------------------------------------------------------ 8-bit rows

@pytest.mark.parametrize("rows,K", [(1, 1), (3, 127), (5, 128), (2, 129), (7, 2047), (4, 2048), (3, 2049),
                                    (2, 8192), (3, 8201), (2, 20000), (1000, 1152)])
@DTYPES
def test_quant_rows_is_exact(rows, K, dtype):
    say("quant", rows, K, NAME[dtype])
    x, _ = rnd(rows * K, (rows, K), 3.0, dtype)
    if rows > 2:
        x[1] = 0
        x[2] *= 2.0 ** -120
    q, s = t2i.quant_rows(x)
    rq, rs = blocks.quant_rows(to_host(x))
    assert np.array_equal(s.cpu().numpy(), rs)
    q = q.cpu().numpy()
    assert q.shape == (rows, (K + 127) // 128 * 128)
    assert np.array_equal(q[:, :K], rq) and not q[:, K:].any()


@DTYPES
def test_quant_rows_ties_and_values_beside_them(dtype):
    """Halves of a row of scale 1, and for other scales the values nearest to every half."""
    half = np.arange(-127, 127) + 0.5
    rows = [np.concatenate([half, [127.0, 0]])]
    for top in (3.0, 0.7, 1e-30, 2.0 ** -125, 3e38, 130.0):
        s = np.float32(np.float32(to_host(dev([top], dtype))[0]) / np.float32(127))
        near = dev((half * np.float64(s)).astype(np.float32), dtype)
        rows.append(np.concatenate([np.clip(to_host(near), -top, top), [top, 0]]))
        up = torch.nextafter(near, torch.full_like(near, 3e38))
        rows.append(np.concatenate([np.clip(to_host(up), -top, top), [top, 0]]))
    x = dev(np.stack(rows).astype(np.float32), dtype)
    q, s = t2i.quant_rows(x)
    rq, rs = blocks.quant_rows(to_host(x))
    assert np.array_equal(s.cpu().numpy(), rs)
    assert np.array_equal(q.cpu().numpy()[:, :256], rq)


@DTYPES
def test_quant_rows_not_finite_rows_strides_and_surroundings(dtype):
    K = 300
    x, _ = rnd(5, (6, K), 1.0, dtype)
    x[1, 299] = float("nan")
    x[3, 0] = float("-inf")
    rq, rs = blocks.quant_rows(to_host(x))
    for extra in (0, 1, 20):   # 20: rows apart by whole 16-byte pieces in both types
        xs, _ = padded(x, extra)
        lib, ldq = t2i.load(), 400
        q = torch.full((7, ldq), 99, dtype=torch.int8, device=DEV)
        s = torch.full((7,), 5.0, device=DEV)
        _lib.check(lib.t2i_op_quant_rows(int(dtype == BF16), 6, K, xs.data_ptr(), xs.stride(0), q.data_ptr(),
                                         ldq, s.data_ptr(), C.c_void_p(torch.cuda.current_stream().cuda_stream)))
        assert np.array_equal(s[:6].cpu().numpy(), rs, equal_nan=True) and s[6] == 5
        assert np.array_equal(q[:6, :K].cpu().numpy(), rq) and not q[:6, K:384].any()
        assert (q[:6, 384:] == 99).all() and (q[6] == 99).all()


# ------------------------------------------------------------------ 8-bit linear layer

def i8_operands(M, N, K, seed=0, wide=0):
    r = np.random.default_rng(seed + M * 31 + N * 7 + K)
    Kp = (K + 127) // 128 * 128
    a, w = np.zeros((M, Kp + wide), np.int8), np.zeros((N, Kp + wide), np.int8)
    a[:, :K], w[:, :K] = r.integers(-127, 128, (M, K)), r.integers(-127, 128, (N, K))
    w[:, K:] = 55    # zeros behind K are needed in one operand only
    sa = r.uniform(0.5, 2, M).astype(np.float32) / 127
    sw = r.uniform(0.5, 2, N).astype(np.float32) / (127 * K ** 0.5)
    return a, sa, w, sw


def i8_bound(acc, b, ref, dtype, epi):
    """acc to fp32, two scalings and the bias: four roundings; then the activation"""
    lin = 4 * E * (np.abs(acc) + (0 if b is None else np.abs(b)))
    if epi in ("gelu", "silu"):
        lin = 1.13 * lin + 2.0 ** -20 * (np.abs(acc) + (0 if b is None else np.abs(b)))
    return U[dtype] * (np.abs(ref) + lin) + lin


I8_SHAPES = [(1, 1, 1), (1, 64, 128), (1, 4608, 1152), (3, 130, 257), (16, 96, 500), (17, 65, 640),
             (33, 1152, 96), (64, 64, 64), (65, 129, 130), (127, 1000, 1151), (130, 512, 4096),
             (257, 300, 1152), (333, 1152, 4096), (520, 2304, 384), (1025, 770, 129), (2100, 1152, 1152)]


@pytest.mark.parametrize("M,N,K", I8_SHAPES)
@DTYPES
def test_linear_i8(M, N, K, dtype):
    say("linear_i8", M, N, K, NAME[dtype])
    a, sa, w, sw = i8_operands(M, N, K)
    d = [dev(v, torch.int8) if v.dtype == np.int8 else dev(v) for v in (a, sa, w, sw)]
    b, rb = rnd(9, (N,), 0.3, dtype)
    acc = blocks.linear_i8(a[:, :K], sa, w[:, :K], sw)
    for epi, bias in (("store", None), ("store", rb), ("gelu", rb), ("silu", rb)):
        ref = acc if bias is None else acc + bias
        if epi != "store":
            ref = blocks.act(epi, ref)
        out = t2i.linear_i8(*d, None if bias is None else b, K=K, epilogue=epi, dtype=dtype)
        assert out.dtype == dtype
        within(out, ref, i8_bound(acc, bias, ref, dtype, epi), (epi, bias is None))


@pytest.mark.parametrize("M,N,K", [(1, 70, 300), (5, 128, 128), (70, 1152, 1152), (300, 260, 700),
                                   (2050, 1152, 256)])
def test_linear_i8_residual_updates(M, N, K):
    a, sa, w, sw = i8_operands(M, N, K, 3)
    d = [dev(v, torch.int8) if v.dtype == np.int8 else dev(v) for v in (a, sa, w, sw)]
    b, rb = rnd(10, (N,), 0.3, BF16)
    gate, rg = rnd(11, (N,), 0.5)
    x0, rx = rnd(12, (M, N), 2.0)
    y = blocks.linear_i8(a[:, :K], sa, w[:, :K], sw, rb)
    for epi, g in (("resid", np.ones(N)), ("resid_gated", rg)):
        for copy in (False, True):
            x, buf = padded(x0, 3)
            cp, cbuf = padded(x0.to(BF16), 3)
            out = t2i.linear_i8(*d, b, K=K, epilogue=epi, resid=x, resid_copy=cp if copy else None,
                                gate=gate if epi == "resid_gated" else None)
            assert out is x
            ref = rx + g * y
            # the layer's bound, the product and the sum
            tol = np.abs(g) * i8_bound(y - rb, rb, y, F32, "store") + 2 * E * (np.abs(g * y) + np.abs(ref))
            within(x, ref, tol, epi)
            assert (buf[:-1, N:] == 7).all() and (buf[-1] == 7).all()
            if copy:
                assert torch.equal(cp, x.to(BF16)) and (cbuf[:-1, N:] == 7).all()


@DTYPES
def test_linear_i8_largest_sums_strides_and_surroundings(dtype):
    # the deepest product of the largest values: 2^31 - 2^14, exact
    K = 131071
    a = np.full((2, 131072), -128, np.int8)
    w = a[:1].repeat(3, 0).copy()
    a[:, K:] = 0
    one = torch.ones(3, device=DEV)
    out = t2i.linear_i8(dev(a, torch.int8), one[:2], dev(w, torch.int8), one, K=K, dtype=F32)
    assert (out == float(128 * 128 * K)).all()
    # operands and outputs inside larger buffers
    M, N, K = 37, 45, 200
    a, sa, w, sw = i8_operands(M, N, K, 5, wide=64)
    ref = blocks.linear_i8(a[:, :K], sa, w[:, :K], sw)
    buf = torch.full((M + 2, N + 3), 7.0, dtype=dtype, device=DEV)
    d = [dev(v, torch.int8) if v.dtype == np.int8 else dev(v) for v in (a, sa, w, sw)]
    _lib.check(t2i.load().t2i_op_linear_i8(
        int(dtype == BF16), 0, M, N, K, d[0].data_ptr(), a.shape[1], d[1].data_ptr(), d[2].data_ptr(),
        w.shape[1], d[3].data_ptr(), None, buf.data_ptr(), N + 3, None, 0, None, None,
        C.c_void_p(torch.cuda.current_stream().cuda_stream)))
    within(buf[:M, :N], ref, i8_bound(ref, None, ref, dtype, "store"))
    assert (buf[:M, N:] == 7).all() and (buf[M:] == 7).all()


def test_linear_i8_not_finite_rows_stay_apart():
    x, _ = rnd(21, (40, 256), 1.0, BF16)
    x[7, 3] = float("inf")
    x[9, 200] = float("nan")
    w, _ = rnd(22, (100, 256), 0.05)
    out = t2i.linear_i8(*t2i.quant_rows(x), *t2i.quant_rows(w), K=256)
    nan = torch.isnan(out)
    assert nan[[7, 9]].all() and nan.sum() == 200


def test_linear_i8_rows_do_not_depend_on_the_batch():
    a, sa, w, sw = i8_operands(700, 1152, 1152, 8)
    d = [dev(v, torch.int8) if v.dtype == np.int8 else dev(v) for v in (a, sa, w, sw)]
    whole = t2i.linear_i8(*d, K=1152, epilogue="gelu")
    for i, n in ((0, 1), (5, 16), (100, 33), (3, 400)):
        assert torch.equal(t2i.linear_i8(d[0][i:i + n], d[1][i:i + n], d[2], d[3], K=1152, epilogue="gelu"),
                           whole[i:i + n])


# ------------------------------------------------------------------ gated feed-forward

def gated_case(M, F, K, dtype, bias, seed=1):
    """(device tensors, the same in float64): x, wg, wu, bg, bu"""
    t = dict(x=rnd(seed, (M, K), 1.0, dtype), wg=rnd(seed + 1, (F, K), K ** -0.5, dtype),
             wu=rnd(seed + 2, (F, K), K ** -0.5, dtype), bg=rnd(seed + 3, (F,), 0.3, dtype),
             bu=rnd(seed + 4, (F,), 0.3, dtype))
    if not bias:
        t["bg"] = t["bu"] = (None, None)
    return {k: v[0] for k, v in t.items()}, {k: v[1] for k, v in t.items()}


def pre_bound(h, K):
    """Error bound of g and u: K products and the bias in fp32"""
    ax = np.abs(h["x"])
    out = []
    for w, b in (("wg", "bg"), ("wu", "bu")):
        out.append((K + 1) * E * (ax @ np.abs(h[w]).T + (0 if h[b] is None else np.abs(h[b]))))
    return out


GATED_SHAPES = [(1, 8, 8), (1, 1152, 1152), (2, 64, 136), (17, 40, 64), (64, 64, 64), (65, 136, 128),
                (130, 256, 192), (333, 1544, 1152), (257, 1000, 264), (700, 128, 4096), (2050, 264, 128)]


@pytest.mark.parametrize("M,F,K", GATED_SHAPES)
@pytest.mark.parametrize("act", ["silu", "gelu"])
@DTYPES
def test_gated_linear(M, F, K, act, dtype):
    say("gated", M, F, K, act, NAME[dtype])
    for bias in (False, True):
        d, h = gated_case(M, F, K, dtype, bias)
        g, u = blocks.gated_pre(**h)
        eg, eu = pre_bound(h, K)
        ref = blocks.gated(act, g, u)
        out, pre = t2i.gated_linear(*d.values(), act=act, save_pre=True)
        a = np.abs(blocks.act(act, g))
        tol = 1.13 * eg * (np.abs(u) + eu) + a * eu + 2.0 ** -20 * np.abs(g * u) + 2 * E * np.abs(ref)
        within(out, ref, tol + U[dtype] * (np.abs(ref) + tol), "out")
        within(pre[:, :F], g, eg + E * (np.abs(g) + eg), "g")
        within(pre[:, F:], u, eu + E * (np.abs(u) + eu), "u")
        if dtype == BF16:   # rounding once: at most half a step of each value
            assert rel_l2(to_host(out), ref) < 2.0 ** -8
        assert torch.equal(t2i.gated_linear(*d.values(), act=act), out)


@pytest.mark.parametrize("M,F,K,extra", [(5, 1, 1, 0), (3, 7, 5, 0), (70, 33, 65, 0), (130, 131, 257, 0),
                                         (130, 132, 260, 0), (130, 131, 260, 0), (130, 132, 257, 0), (70, 36, 68, 4), (70, 36, 68, 1), (300, 700, 333, 2),
                                         (2100, 12, 20, 0)])
def test_gated_linear_f32_any_width(M, F, K, extra):
    """Widths and strides that are no multiples of 16 bytes, and of 16 but not of 32."""
    d, h = gated_case(M, F, K, F32, True, 30)
    d["x"] = padded(d["x"], extra)[0]
    g, u = blocks.gated_pre(**h)
    eg, eu = pre_bound(h, K)
    ref = blocks.gated("silu", g, u)
    out, pre = t2i.gated_linear(*d.values(), save_pre=True)
    tol = 1.13 * eg * (np.abs(u) + eu) + np.abs(blocks.act("silu", g)) * eu + 2.0 ** -20 * np.abs(g * u) + 3 * E * np.abs(ref)
    within(out, ref, tol)
    dout, hd = rnd(31, (M, F))
    check_backward(F32, "silu", d, h, pre, dout, hd)


def check_backward(dtype, act, d, h, pre, dout, hdout):
    M, K = h["x"].shape
    F = h["wg"].shape[0]
    hp = to_host(pre)
    g, u = hp[:, :F], hp[:, F:]
    r = blocks.gated_grads(act, hdout, h["x"], h["wg"], h["wu"], g, u)
    got = t2i.gated_linear_backward(dout, d["x"], d["wg"], d["wu"], pre, act=act, bias=True)
    # dg, du in fp32 (the activation's few E, relative to dout u (1 + |g|) and
    # dout a), then their one rounding to the type
    fg = 2.0 ** -20 * np.abs(hdout * u) * (1 + np.abs(g))
    fu = 2.0 ** -20 * np.abs(hdout * g)
    eg, eu = fg + U[dtype] * (np.abs(r["dg"]) + fg), fu + U[dtype] * (np.abs(r["du"]) + fu)
    ag, au = np.abs(r["dg"]) + eg, np.abs(r["du"]) + eu
    wg, wu, ax = np.abs(h["wg"]), np.abs(h["wu"]), np.abs(h["x"])
    tol = dict(dx=eg @ wg + eu @ wu + 2 * F * E * (ag @ wg + au @ wu),
               dwg=eg.T @ ax + M * E * (ag.T @ ax), dwu=eu.T @ ax + M * E * (au.T @ ax),
               dbg=fg.sum(0) + M * E * ag.sum(0), dbu=fu.sum(0) + M * E * au.sum(0))
    for name, t in zip(("dx", "dwg", "dwu", "dbg", "dbu"), got):
        assert t.dtype == dtype
        within(t, r[name], tol[name] + U[dtype] * (np.abs(r[name]) + tol[name]), name)
        if name in ("dx", "dwg", "dwu") and dtype == BF16 and M * F > 64:
            # two independent roundings of 2^-8 / sqrt(3) at most: well inside 2^-7
            assert rel_l2(to_host(t), r[name]) < 2.0 ** -7, name
    return got


@pytest.mark.parametrize("M,F,K", GATED_SHAPES)
@pytest.mark.parametrize("act", ["silu", "gelu"])
@DTYPES
def test_gated_linear_backward(M, F, K, act, dtype):
    say("gated backward", M, F, K, act, NAME[dtype])
    d, h = gated_case(M, F, K, dtype, True, 40)
    pre, _ = rnd(50, (M, 2 * F), 1.5)
    dout, hd = rnd(51, (M, F), 1.0, dtype)
    got = check_backward(dtype, act, d, h, pre, dout, hd)
    # each gradient alone is the same gradient
    args = (dout, d["x"], d["wg"], d["wu"], pre)
    dx = t2i.gated_linear_backward(*args, act=act, need_dw=False)
    dw = t2i.gated_linear_backward(*args, act=act, need_dx=False)
    assert torch.equal(dx[0], got[0]) and dx[1] is None and dx[3] is None
    assert torch.equal(dw[1], got[1]) and torch.equal(dw[2], got[2]) and dw[0] is None


@DTYPES
def test_gated_extreme_preactivations(dtype):
    """Pre-activations whose exponentials overflow or vanish: limits, no NaN."""
    vals = [-1e30, -3e4, -100.0, -20.0, -0.0, 0.0, 1e-30, 20.0, 100.0, 3e4, 1e30, 0.5]
    M, F, K = len(vals), 8, 8
    pre = torch.ones((M, 2 * F), device=DEV)
    pre[:, :F] = dev(np.array(vals, np.float32))[:, None]
    d, h = gated_case(M, F, K, dtype, True, 60)
    dout = torch.ones((M, F), dtype=dtype, device=DEV)
    for act in ("silu", "gelu"):
        with np.errstate(over="ignore", invalid="ignore"):
            g = to_host(pre)[:, :F]
            t = torch.from_numpy(g).requires_grad_()
            f = torch.nn.functional.silu(t) if act == "silu" else torch.nn.functional.gelu(t.clamp(-1e4, 1e4), approximate="tanh")
            da, = torch.autograd.grad(f.sum(), t)
        da = np.where(np.abs(g) > 1e4, (g > 0).astype(np.float64), da.numpy())
        # the identity as weights: dx = dg + du
        eye = torch.eye(8, dtype=dtype, device=DEV)
        zero = torch.zeros_like(eye)
        dx = t2i.gated_linear_backward(dout, d["x"], eye, zero, pre, act=act, need_dw=False)[0]
        within(dx, da, U[dtype] * np.abs(da) + 2.0 ** -20 * (1 + np.minimum(np.abs(da * g), 10)), act)


def test_gated_backward_against_differences():
    """The kernels' gradient against differences of the kernels' own forward pass (fp32)."""
    M, F, K = 9, 24, 16
    d, _ = gated_case(M, F, K, F32, True, 70)
    dout, _ = rnd(75, (M, F))
    _, pre = t2i.gated_linear(*d.values(), act="gelu", save_pre=True)
    grads = t2i.gated_linear_backward(dout, d["x"], d["wg"], d["wu"], pre, act="gelu", bias=True)
    for (name, t), g in zip(d.items(), grads):
        step, _ = rnd(80 + len(name), tuple(t.shape))
        loss = []
        for sign in (1, -1):
            p = dict(d)
            p[name] = t + sign * 2.0 ** -7 * step
            loss.append((t2i.gated_linear(*p.values(), act="gelu").double() * dout.double()).sum().item())
        num, ana = (loss[0] - loss[1]) * 2 ** 6, (g.double() * step.double()).sum().item()
        # h^2 / 6 = 1e-5 of a third derivative of the gradient's size; fp32 noise of 216
        # outputs over h: 2^-24 * 15 * 128; both far below 2 % of |gradient| |step|
        scale = g.double().norm().item() * step.double().norm().item() / (t.numel() ** 0.5)
        assert abs(num - ana) < 0.02 * scale + 1e-3, name


@DTYPES
def test_gated_strides_and_surroundings(dtype):
    M, F, K = 70, 72, 136
    d, h = gated_case(M, F, K, dtype, True, 90)
    ref, rpre = t2i.gated_linear(*d.values(), save_pre=True)
    w2, _ = padded(torch.cat([d["wg"], d["wu"]]), 8)      # one [2F, K] matrix of wider rows
    x, _ = padded(d["x"], 24)
    out = torch.full((M + 1, F + 8), 7.0, dtype=dtype, device=DEV)
    pre = torch.full((M + 1, 2 * F + 8), 7.0, device=DEV)
    st = C.c_void_p(torch.cuda.current_stream().cuda_stream)
    dt = int(dtype == BF16)
    _lib.check(t2i.load().t2i_op_gated_linear(
        dt, _lib.T2I_EPI_SILU, M, F, K, x.data_ptr(), K + 24, w2.data_ptr(), w2[F:].data_ptr(), K + 8,
        d["bg"].data_ptr(), d["bu"].data_ptr(), out.data_ptr(), F + 8, pre.data_ptr(), 2 * F + 8, st))
    assert torch.equal(out[:M, :F], ref) and (out[:M, F:] == 7).all() and (out[M] == 7).all()
    assert torch.equal(pre[:M, :2 * F], rpre) and (pre[:M, 2 * F:] == 7).all() and (pre[M] == 7).all()
    dout, _ = rnd(95, (M, F), 1.0, dtype)
    want = t2i.gated_linear_backward(dout, d["x"], d["wg"], d["wu"], rpre, bias=True)
    do, _ = padded(dout, 16)
    dx = torch.full((M + 1, K + 8), 7.0, dtype=dtype, device=DEV)
    dw = torch.full((2 * F + 1, K + 16), 7.0, dtype=dtype, device=DEV)
    n = t2i.load().t2i_op_gated_linear_backward_ws_bytes(dt, M, F, K)
    for fill in (0, 255):   # whatever the workspace held
        ws = torch.full((n,), fill, dtype=torch.uint8, device=DEV)
        _lib.check(t2i.load().t2i_op_gated_linear_backward(
            dt, _lib.T2I_EPI_SILU, M, F, K, x.data_ptr(), K + 24, w2.data_ptr(), w2[F:].data_ptr(), K + 8,
            pre.data_ptr(), 2 * F + 8, do.data_ptr(), F + 16, dx.data_ptr(), K + 8, dw.data_ptr(),
            dw[F:].data_ptr(), K + 16, None, None, ws.data_ptr(), n, st))
        assert torch.equal(dx[:M, :K], want[0]) and (dx[:M, K:] == 7).all() and (dx[M] == 7).all()
        assert torch.equal(dw[:F, :K], want[1]) and torch.equal(dw[F:2 * F, :K], want[2])
        assert (dw[:, K:] == 7).all() and (dw[2 * F] == 7).all()


def inside_nan(t, rows=70):
    """t as the first rows and columns of a buffer of NaN, `rows` rows of it behind t."""
    buf = torch.full((t.shape[0] + rows, t.shape[1] + 8), float("nan"), dtype=t.dtype, device=DEV)
    buf[:t.shape[0], :t.shape[1]] = t
    return buf[:t.shape[0], :t.shape[1]]


@pytest.mark.parametrize("M,F,K", [(2, 8, 1256), (3, 72, 40), (33, 40, 72), (65, 104, 200), (130, 264, 136)])
@DTYPES
def test_gated_reads_nothing_behind_its_operands(M, F, K, dtype):
    d, h = gated_case(M, F, K, dtype, True, 110)
    for name in ("x", "wg", "wu"):
        d[name] = inside_nan(d[name])
    out, pre = t2i.gated_linear(*d.values(), save_pre=True)
    assert torch.isfinite(out).all() and torch.isfinite(pre).all()
    dout, hd = rnd(111, (M, F), 1.0, dtype)
    check_backward(dtype, "silu", d, h, inside_nan(pre), inside_nan(dout), hd)


def test_gated_not_finite_values_stay_where_they_belong():
    M, F, K = 70, 72, 136
    d, _ = gated_case(M, F, K, BF16, False, 100)
    d["x"][69, 135] = float("nan")
    d["wg"][71, 0] = float("inf")
    out, pre = t2i.gated_linear(*d.values(), save_pre=True)
    bad = ~torch.isfinite(pre[:, :F])
    assert bad[69].all() and bad[:, 71].all() and bad.sum() == M + F - 1
    assert torch.isfinite(out[:69, :71]).all()
    # gradients: row 69 of x spoils every element of dW through its NaN column only
    d, h = gated_case(M, F, K, BF16, False, 100)
    pre, _ = rnd(101, (M, 2 * F))
    dout, _ = rnd(102, (M, F), 1.0, BF16)
    clean = t2i.gated_linear_backward(dout, d["x"], d["wg"], d["wu"], pre)
    d["x"][69, 135] = float("nan")
    d["wg"][71, 130] = float("nan")
    got = t2i.gated_linear_backward(dout, d["x"], d["wg"], d["wu"], pre)
    for a, b, col in ((clean[0], got[0], 130), (clean[1], got[1], 135), (clean[2], got[2], 135)):
        keep = torch.ones(K, dtype=torch.bool, device=DEV)
        keep[col] = False
        assert torch.isnan(b[:, col]).all() and torch.equal(a[:, keep], b[:, keep])


# ------------------------------------------------------------------ every tile, long rows

def tile_of(op, dtype, M, F, K):
    """(rows, columns, workgroups per CU, slices or groups of waves) that a product takes"""
    v = [C.c_int() for _ in range(4)]
    assert t2i.load().t2i_test_block_tile(op, int(dtype == BF16), M, F, K, *map(C.byref, v))
    return tuple(x.value for x in v)


def some(n, seed):
    """A few indices below n, the first and the last among them."""
    r = np.random.default_rng(seed)
    return np.unique(np.concatenate([[0, n - 1], r.integers(0, n, min(n, 40))]))


@pytest.mark.parametrize("M,N,K,tile", [
    (20, 72, 72, (32, 128, 2)), (30, 16500, 72, (32, 128, 1)), (8200, 136, 72, (64, 128, 2)),
    (8200, 520, 72, (64, 128, 3)), (8200, 264, 2056, (128, 128, 1)), (8200, 520, 2056, (128, 128, 2)),
    (4090, 4090, 4104, (256, 256, 1)), (17, 72, 521, (16, 32, 2, 4)), (33, 3000, 650, (16, 32, 2, 4)),
    (1, 41, 7447, (16, 32, 2, 4)), (200, 1033, 650, (32, 64, 2, 2)), (130, 2056, 1100, (32, 64, 2, 2))])
def test_linear_i8_on_every_tile(M, N, K, tile):
    assert tile_of(0, BF16, M, N, K) == (*tile, 1)[:4]
    a, sa, w, sw = i8_operands(M, N, K, 120)
    d = [dev(v, torch.int8) if v.dtype == np.int8 else dev(v) for v in (a, sa, w, sw)]
    b, rb = rnd(121, (N,), 0.3, BF16)
    i = some(M, 1)
    # (an exact product in float64: whole numbers below 2^53)
    acc = (a[i, :K].astype(np.float64) @ w[:, :K].astype(np.float64).T) * sa[i, None].astype(np.float64) * sw
    for dtype in (BF16, F32):
        bias = b.to(dtype)
        for epi in ("store", "gelu"):
            ref = acc + rb if epi == "store" else blocks.act(epi, acc + rb)
            out = t2i.linear_i8(*d, bias, K=K, epilogue=epi, dtype=dtype)
            within(out[torch.from_numpy(i).to(DEV)], ref, i8_bound(acc, rb, ref, dtype, epi), (epi, dtype))
    x0, _ = rnd(122, (M, N), 2.0)
    gate, rg = rnd(123, (N,), 0.5)
    x = t2i.linear_i8(*d, b, K=K, epilogue="resid_gated", resid=x0.clone(), gate=gate)
    y = acc + rb
    ref = to_host(x0[torch.from_numpy(i).to(DEV)]) + rg * y
    within(x[torch.from_numpy(i).to(DEV)], ref,
           np.abs(rg) * i8_bound(acc, rb, y, F32, "store") + 2 * E * (np.abs(rg * y) + np.abs(ref)), "resid")


@pytest.mark.parametrize("M,F,K,dtype,tile", [
    (20, 72, 72, BF16, (32, 128, 2)), (30, 8200, 72, BF16, (32, 128, 1)), (8200, 72, 72, BF16, (64, 128, 2)),
    (8200, 136, 72, BF16, (64, 128, 3)), (8200, 136, 520, BF16, (128, 128, 1)),
    (8200, 264, 520, BF16, (128, 128, 2)), (8200, 520, 2056, BF16, (256, 256, 1)),
    (300, 200, 72, F32, (32, 64, 1)), (300, 199, 71, F32, (32, 64, 1)), (8200, 1032, 72, F32, (64, 64, 1)), (8200, 1031, 71, F32, (64, 64, 1)),
    (1032, 1544, 72, F32, (128, 128, 1)), (1032, 1543, 71, F32, (128, 128, 1)),
    (17, 40, 264, BF16, (16, 32, 2, 4)), (1, 72, 2056, BF16, (16, 32, 2, 4)), (33, 520, 328, BF16, (16, 32, 2, 4)),
    (200, 520, 264, BF16, (32, 64, 2, 2)), (70, 4104, 328, BF16, (32, 64, 2, 2)),
    (5, 41, 131, F32, (16, 32, 2, 4)), (17, 40, 164, F32, (16, 32, 2, 4)), (40, 521, 2049, F32, (16, 32, 2, 4)),
    (130, 1032, 264, F32, (32, 64, 1, 2)), (130, 1033, 299, F32, (32, 64, 1, 2))])
def test_gated_linear_on_every_tile(M, F, K, dtype, tile):
    assert tile_of(1, dtype, M, F, K) == (*tile, 1)[:4]
    d, h = gated_case(M, F, K, dtype, True, 130)
    out, pre = t2i.gated_linear(*d.values(), act="silu", save_pre=True)
    i = some(M, 2)
    it = torch.from_numpy(i).to(DEV)
    h["x"] = h["x"][i]
    g, u = blocks.gated_pre(**h)
    eg, eu = pre_bound(h, K)
    ref = blocks.gated("silu", g, u)
    tol = 1.13 * eg * (np.abs(u) + eu) + np.abs(blocks.act("silu", g)) * eu + 2.0 ** -20 * np.abs(g * u) + 2 * E * np.abs(ref)
    within(out[it], ref, tol + U[dtype] * (np.abs(ref) + tol))
    within(pre[it], np.concatenate([g, u], 1), np.concatenate([eg, eu], 1) + E * np.abs(np.concatenate([g, u], 1)))


@pytest.mark.parametrize("op,M,F,K,dtype,tile", [
    ("dx", 20, 72, 72, BF16, (32, 128, 2, 1)), ("dx", 20, 520, 72, BF16, (32, 128, 2, 5)),
    ("dx", 8200, 72, 200, BF16, (64, 128, 2, 1)), ("dx", 4100, 1032, 72, BF16, (64, 128, 2, 4)),
    ("dx", 8200, 72, 520, BF16, (64, 128, 3, 1)), ("dx", 4100, 4104, 72, BF16, (64, 128, 3, 10)),
    ("dx", 4100, 1032, 520, BF16, (128, 128, 1, 1)), ("dx", 2050, 2056, 520, BF16, (128, 128, 1, 3)),
    ("dx", 8200, 520, 520, BF16, (128, 128, 2, 1)), ("dx", 4100, 4104, 520, BF16, (128, 128, 2, 3)),
    ("dx", 8200, 2056, 1032, BF16, (256, 256, 1, 1)), ("dx", 2050, 8200, 2056, BF16, (256, 256, 1, 3)),
    ("dx", 20, 72, 72, F32, (32, 64, 1, 1)), ("dx", 20, 264, 72, F32, (32, 64, 1, 5)),
    ("dx", 8200, 72, 2056, F32, (64, 64, 1, 1)), ("dx", 8200, 71, 2055, F32, (64, 64, 1, 1)),
    ("dx", 2056, 72, 1544, F32, (128, 128, 1, 1)), ("dx", 2056, 71, 1543, F32, (128, 128, 1, 1)),
    ("dx", 4100, 520, 200, F32, (32, 64, 1, 1)), ("dx", 4100, 521, 203, F32, (32, 64, 1, 1)),
    ("dx", 1032, 1032, 1032, F32, (128, 128, 1, 3)), ("dx", 1032, 1031, 1033, F32, (128, 128, 1, 3)),
    ("dx", 520, 520, 200, F32, (64, 64, 1, 6)), ("dx", 520, 519, 201, F32, (64, 64, 1, 6)),
    ("dx", 77, 1031, 333, F32, (32, 64, 1, 14)), ("dx", 70, 1031, 65, F32, (32, 64, 1, 14)),
    ("dw", 20, 72, 72, BF16, (32, 128, 2, 1)), ("dw", 2050, 72, 72, BF16, (32, 128, 2, 9)),
    ("dw", 20, 8200, 72, BF16, (64, 128, 2, 1)), ("dw", 2050, 2056, 72, BF16, (64, 128, 2, 4)),
    ("dw", 20, 8200, 200, BF16, (64, 128, 3, 1)), ("dw", 4100, 4104, 72, BF16, (64, 128, 3, 5)),
    ("dw", 2050, 2056, 520, BF16, (128, 128, 1, 1)), ("dw", 4100, 1032, 520, BF16, (128, 128, 1, 3)),
    ("dw", 130, 8200, 1032, BF16, (128, 128, 2, 1)), ("dw", 8200, 2056, 520, BF16, (128, 128, 2, 3)),
    ("dw", 2050, 8200, 520, BF16, (256, 256, 1, 1)), ("dw", 20, 72, 72, F32, (64, 64, 1, 1)),
    ("dw", 520, 72, 72, F32, (64, 64, 1, 5)), ("dw", 20, 8200, 72, F32, (64, 64, 1, 1)),
    ("dw", 20, 8199, 71, F32, (64, 64, 1, 1)), ("dw", 72, 1032, 1544, F32, (128, 128, 1, 1)),
    ("dw", 72, 1031, 1543, F32, (128, 128, 1, 1)), ("dw", 1030, 2056, 200, F32, (128, 128, 1, 3)),
    ("dw", 1030, 2055, 203, F32, (128, 128, 1, 3)), ("dw", 3001, 131, 77, F32, (64, 64, 1, 16))])
def test_gated_gradients_on_every_tile(op, M, F, K, dtype, tile):
    assert tile_of(2 if op == "dx" else 3, dtype, M, F, K) == tile
    say(op, M, F, K, NAME[dtype], tile)
    d, h = gated_case(M, F, K, dtype, False, 140)
    pre, hp = rnd(141, (M, 2 * F), 1.5)
    dout, hd = rnd(142, (M, F), 1.0, dtype)
    got = t2i.gated_linear_backward(dout, d["x"], d["wg"], d["wu"], pre, act="gelu", need_dx=op == "dx",
                                    need_dw=op == "dw")
    i = some(M if op == "dx" else F, 3)
    it = torch.from_numpy(i).to(DEV)
    g, u = hp[:, :F], hp[:, F:]
    if op == "dx":
        g, u, hd = g[i], u[i], hd[i]
    else:
        g, u, hd = g[:, i], u[:, i], hd[:, i]
    dg, du = hd * u * blocks.act_grad("gelu", g), hd * blocks.act("gelu", g)
    fg, fu = 2.0 ** -20 * np.abs(hd * u) * (1 + np.abs(g)), 2.0 ** -20 * np.abs(hd * g)
    eg, eu = fg + U[dtype] * (np.abs(dg) + fg), fu + U[dtype] * (np.abs(du) + fu)
    if op == "dx":
        cases = [(got[0], dg @ h["wg"] + du @ h["wu"], eg @ np.abs(h["wg"]) + eu @ np.abs(h["wu"]) +
                  2 * F * E * (np.abs(dg) @ np.abs(h["wg"]) + np.abs(du) @ np.abs(h["wu"])))]
    else:
        ax = np.abs(h["x"])
        cases = [(got[1], dg.T @ h["x"], eg.T @ ax + M * E * (np.abs(dg).T @ ax)),
                 (got[2], du.T @ h["x"], eu.T @ ax + M * E * (np.abs(du).T @ ax))]
    for t, ref, tol in cases:
        within(t[it], ref, tol + U[dtype] * (np.abs(ref) + tol), op)
        assert rel_l2(to_host(t[it]), ref) < (2.0 ** -7 if dtype == BF16 else 2.0 ** -17)


@pytest.mark.parametrize("M,F,K", [(5, 40, 37), (33, 130, 70), (70, 129, 132), (200, 1032, 264), (130, 72, 513),
                                   (1030, 300, 203), (1032, 1544, 72)])
@pytest.mark.parametrize("at", [1, 2, 3])
def test_gated_f32_rows_at_any_address(M, F, K, at):
    """Operands cut out of wider matrices of NaN, off 16 bytes: the contiguous operands'
    results bit for bit (the same sums in the same order)."""
    say("any address", M, F, K, at)
    d, _ = gated_case(M, F, K, F32, True, 160)
    dout, _ = rnd(161, (M, F))

    def cut(t):
        wide = torch.full((t.shape[0], t.shape[1] + 5), float("nan"), device=DEV)
        v = wide[:, at:at + t.shape[1]]
        v.copy_(t)
        return v

    def both(x, wg, wu, dh):
        h, pre = t2i.gated_linear(x, wg, wu, d["bg"], d["bu"], act="gelu", save_pre=True)
        return [h, pre, *t2i.gated_linear_backward(dh, x, wg, wu, pre, act="gelu", bias=True)]

    a = both(d["x"], d["wg"], d["wu"], dout)
    b = both(cut(d["x"]), cut(d["wg"]), cut(d["wu"]), cut(dout))
    for n, u, v in zip(("h", "pre", "dx", "dwg", "dwu", "dbg", "dbu"), a, b):
        assert torch.isfinite(u).all() and torch.equal(u, v), n


def test_rows_far_apart():
    """Offsets past 32 bits: rows just below 8 MiB apart in tensors of more than 2 GiB."""
    M, F, K, wide = 300, 264, 72, 2 ** 22 - 8
    d, _ = gated_case(M, F, K, BF16, False, 150)
    dout, _ = rnd(151, (M, F), 1.0, BF16)
    out, pre = t2i.gated_linear(*d.values(), save_pre=True)
    want = t2i.gated_linear_backward(dout, d["x"], d["wg"], d["wu"], pre)
    x = torch.empty((M, wide), dtype=BF16, device=DEV)[:, :K]
    w = torch.empty((2 * F, wide), dtype=BF16, device=DEV)[:, :K]
    x.copy_(d["x"])
    w[:F], w[F:] = d["wg"], d["wu"]
    got = t2i.gated_linear(x, w[:F], w[F:], save_pre=True)
    assert torch.equal(got[0], out) and torch.equal(got[1], pre)
    for a, b in zip(t2i.gated_linear_backward(dout, x, w[:F], w[F:], pre)[:3], want):
        assert torch.equal(a, b)
    q, s = t2i.quant_rows(x)
    q0, s0 = t2i.quant_rows(d["x"])
    assert torch.equal(q, q0) and torch.equal(s, s0)
    del x, w, got
    big = torch.zeros((M, 2 ** 23 - 16), dtype=torch.int8, device=DEV)
    big[:, :128] = q
    wq, ws = t2i.quant_rows(d["wg"])
    assert torch.equal(t2i.linear_i8(big, s, wq, ws, K=K), t2i.linear_i8(q, s, wq, ws, K=K))
    del big
    heads = torch.empty((M, wide), dtype=BF16, device=DEV)[:, :K].unflatten(1, (1, 72))
    heads.copy_(d["x"].unflatten(1, (1, 72)))
    near = d["x"].unflatten(1, (1, 72))
    assert torch.equal(t2i.qk_norm_rope(heads, near)[0], t2i.qk_norm_rope(near, near)[0])
    for a, b in zip(t2i.qk_norm_rope_backward(heads, near, heads, near), t2i.qk_norm_rope_backward(near, near, near, near)):
        assert a is b or torch.equal(a, b)


# ------------------------------------------------------------------ query / key norm with rotation

def qk_case(rows, hq, hk, d, dtype, pairing, seed=1, fused=True):
    r = np.random.default_rng(seed + rows * 13 + d)
    buf, hb = rnd(seed + rows + d, (rows, (hq + hk) * d + 16), 2.0, dtype)
    if fused:
        q, k = buf[:, :hq * d].unflatten(1, (hq, d)), buf[:, hq * d:(hq + hk) * d].unflatten(1, (hk, d))
    else:
        q = buf[:, :hq * d].contiguous().view(rows, hq, d)
        k = buf[:, hq * d:(hq + hk) * d].contiguous().view(rows, hk, d)
    wq, wk = rnd(seed + 2, (d,), 1.0, dtype)[0], rnd(seed + 3, (d,), 1.0, dtype)[0]
    n_pos = 2 * rows + 1
    ang = r.uniform(-1e3, 1e3, (n_pos, d // 2))
    table = dev(np.stack([np.cos(ang), np.sin(ang)], -1).astype(np.float32))
    pos = r.integers(0, n_pos, rows).astype(np.int32)
    pos[r.random(rows) < 0.2] = -1
    return q, k, wq, wk, dict(table=table, pos=dev(pos, torch.int32), pairing=pairing)


def host_rot(rot):
    return dict(table=to_host(rot["table"]), pos=rot["pos"].cpu().numpy(), pairing=rot["pairing"])


QK_SHAPES = [(1, 1, 1, 8, "pairs"), (1, 32, 8, 128, "halves"), (3, 2, 1, 16, "halves"), (5, 3, 3, 24, "pairs"),
             (7, 16, 16, 72, "pairs"), (33, 4, 2, 48, "halves"), (100, 5, 1, 64, "pairs"),
             (257, 24, 24, 128, "pairs"), (300, 6, 3, 80, "halves"), (64, 2, 2, 256, "halves"),
             (65, 3, 1, 136, "pairs"), (2500, 16, 4, 64, "halves"), (4100, 16, 16, 72, "pairs")]


@pytest.mark.parametrize("rows,hq,hk,d,pairing", QK_SHAPES)
@DTYPES
def test_qk_norm_rope(rows, hq, hk, d, pairing, dtype):
    say("qk", rows, hq, hk, d, pairing, NAME[dtype])
    q, k, wq, wk, rot = qk_case(rows, hq, hk, d, dtype, pairing)
    eps = 1e-3
    got = t2i.qk_norm_rope(q, k, wq, wk, eps=eps, **rot)
    hr = host_rot(rot)
    for x, w, o in ((q, wq, got[0]), (k, wk, got[1])):
        hx, hw = to_host(x), to_host(w)
        ref = blocks.qk_norm_rope(hx, hw, eps, **hr)
        # the mean of d squares (d / 8 + 4 sums in turn), root, two products, rotation
        # (of the pair's norm, which bounds what the rotation mixes)
        mix = np.sqrt(pair_energy(blocks.head_norm(hx, hw, eps), pairing))
        tol = (d / 16 + 12) * E * 2 * np.maximum(mix, np.abs(ref))
        within(o, ref, tol + U[dtype] * (np.abs(ref) + tol))


def pair_energy(n, pairing):
    """a^2 + b^2 of each element's pair"""
    d = n.shape[-1]
    if pairing == "pairs":
        return np.repeat((n.reshape(*n.shape[:-1], d // 2, 2) ** 2).sum(-1), 2, -1)
    e = n[..., :d // 2] ** 2 + n[..., d // 2:] ** 2
    return np.concatenate([e, e], -1)


@pytest.mark.parametrize("rows,hq,hk,d,pairing", QK_SHAPES)
@DTYPES
def test_qk_norm_rope_backward(rows, hq, hk, d, pairing, dtype):
    say("qk backward", rows, hq, hk, d, pairing, NAME[dtype])
    q, k, wq, wk, rot = qk_case(rows, hq, hk, d, dtype, pairing, 5)
    dq, hdq = rnd(6, (rows, hq, d), 1.0, dtype)
    dk, hdk = rnd(7, (rows, hk, d), 1.0, dtype)
    eps, hr = 1e-3, host_rot(rot)
    got = t2i.qk_norm_rope_backward(dq, dk, q, k, wq, wk, eps=eps, **rot)
    for i, (x, w, dy) in enumerate(((q, wq, hdq), (k, wk, hdk))):
        hx, hw = to_host(x), to_host(w)
        dx, dw = blocks.qk_norm_rope_grads(dy, hx, hw, eps, **hr)
        r = 1 / np.sqrt((hx * hx).mean(-1, keepdims=True) + eps)
        n, mix = hx * r, np.sqrt(pair_energy(dy, pairing))   # |R^T dy| at most
        # dn, then the mean over the head of |dn n|: d products more
        size = mix * np.abs(hw)
        tol = 2 * (d / 16 + 16) * E * r * (size + np.abs(n) * (size * np.abs(n)).mean(-1, keepdims=True))
        within(got[i], dx, tol + U[dtype] * (np.abs(dx) + tol), "dx")
        # every term a few roundings, the fp32 sums over at most rows heads terms
        # in runs: bounded by (rows heads / 1024 + 64) in turn
        tol = ((rows * (hq + hk) / 512 + 64 + d / 16) * E) * (mix * np.abs(n)).sum((0, 1))
        within(got[2 + i], dw, tol + U[dtype] * (np.abs(dw) + tol), "dw")


@DTYPES
def test_qk_variants(dtype):
    """In place, no weights, no rotation, positions by row, queries alone."""
    q, k, wq, wk, rot = qk_case(37, 4, 2, 64, dtype, "halves", 9)
    both = t2i.qk_norm_rope(q, k, wq, wk, **rot)
    one = torch.ones_like(wq)
    assert all(torch.equal(a, b) for a, b in zip(t2i.qk_norm_rope(q, k, **rot), t2i.qk_norm_rope(q, k, one, one, **rot)))
    still = dict(rot, pos=torch.full_like(rot["pos"], -5))
    assert all(torch.equal(a, b) for a, b in zip(t2i.qk_norm_rope(q, k, wq, wk), t2i.qk_norm_rope(q, k, wq, wk, **still)))
    byrow = dict(rot, pos=torch.arange(37, dtype=torch.int32, device=DEV))
    assert all(torch.equal(a, b) for a, b in zip(t2i.qk_norm_rope(q, k, wq, wk, **dict(rot, pos=None)),
                                                 t2i.qk_norm_rope(q, k, wq, wk, **byrow)))
    alone, none = t2i.qk_norm_rope(q, k[:, :0], wq, wk, **rot)
    assert torch.equal(alone, both[0]) and none.shape == (37, 0, 64)
    none, alone = t2i.qk_norm_rope(q[:, :0], k, wq, wk, **rot)
    assert torch.equal(alone, both[1])
    g = t2i.qk_norm_rope_backward(*both, q, k, wq, wk, **rot)
    g1 = t2i.qk_norm_rope_backward(both[0], k[:, :0], q, k[:, :0], wq, None, **rot)
    assert torch.equal(g1[0], g[0]) and g1[3] is None
    buf = q._base.clone() if q._base is not None else None
    qi, ki = t2i.qk_norm_rope(q, k, wq, wk, inplace=True, **rot)
    assert qi is q and ki is k and torch.equal(q, both[0]) and torch.equal(k, both[1])
    if buf is not None:
        assert torch.equal(q._base[:, -16:], buf[:, -16:])   # columns behind the heads


@DTYPES
def test_qk_positions_behind_the_table_and_not_finite_heads(dtype):
    q, k, wq, wk, rot = qk_case(9, 2, 2, 32, dtype, "pairs", 11)
    clean = t2i.qk_norm_rope(q, k, wq, wk, **rot)
    rot["pos"][4] = rot["table"].shape[0]
    rot["pos"][6] = 2 ** 31 - 1
    q[2, 1, 5] = float("nan")
    got = t2i.qk_norm_rope(q, k, wq, wk, **rot)
    for c, o in zip(clean, got):
        assert torch.isnan(o[[4, 6]]).all()
        keep = torch.tensor([0, 1, 3, 5, 7, 8], device=DEV)
        assert torch.equal(o[keep], c[keep])
    assert torch.isnan(got[0][2, 1]).all() and torch.equal(got[0][2, 0], clean[0][2, 0])
    assert torch.equal(got[1][2], clean[1][2])
    z = t2i.qk_norm_rope(torch.zeros_like(q), torch.zeros_like(k), wq, wk, **dict(rot, pos=None))
    assert not z[0].any() and not z[1].any()


def test_qk_backward_against_differences():
    q, k, wq, wk, rot = qk_case(6, 3, 2, 32, F32, "halves", 13, fused=False)
    w = [rnd(14 + i, tuple(t.shape))[0] for i, t in enumerate((q, k))]
    args = [q, k, wq, wk]
    grads = t2i.qk_norm_rope_backward(*w, *args, **rot)
    for i, g in enumerate(grads):
        step, _ = rnd(17 + i, tuple(args[i].shape))
        loss = []
        for sign in (1, -1):
            p = list(args)
            p[i] = args[i] + sign * 2.0 ** -7 * step
            o = t2i.qk_norm_rope(*p, **rot)
            loss.append(sum((a.double() * b.double()).sum().item() for a, b in zip(o, w)))
        num, ana = (loss[0] - loss[1]) * 2 ** 6, (g.double() * step.double()).sum().item()
        scale = g.double().norm().item() * step.double().norm().item() / g.numel() ** 0.5
        assert abs(num - ana) < 0.02 * scale + 1e-3, i   # as for the gated block


# ------------------------------------------------------------------ streams, graphs, refusals, a block of them

def chain(p, x, resid, rot, segs):
    """A transformer block from the operators: 8-bit qkv, q/k norm with rotation,
    attention, 8-bit output with the residual, LN-modulate, gated feed-forward, 8-bit
    second projection with the gated residual.  Returns the residual stream and q."""
    lib, st = t2i.load(), C.c_void_p(torch.cuda.current_stream().cuda_stream)
    rows, D = x.shape
    H, d = p["H"], p["d"]
    qkv = t2i.linear_i8(*t2i.quant_rows(x), *p["wqkv"], p["bqkv"], K=D)
    q, k = qkv[:, :D].unflatten(1, (H, d)), qkv[:, D:2 * D].unflatten(1, (H, d))
    t2i.qk_norm_rope(q, k, p["nq"], p["nk"], inplace=True, **rot)
    ldv = (rows + 63) // 64 * 64
    vt = torch.zeros((D, ldv), dtype=x.dtype, device=DEV)
    vt[:, :rows] = qkv[:, 2 * D:].t()
    o = torch.zeros_like(x)
    arr = lambda v: (C.c_int32 * len(v))(*v)  # noqa: E731
    s, n = arr([a for a, _ in segs]), arr([b for _, b in segs])
    _lib.check(lib.t2i_op_attention(_lib.T2I_BF16, H, d, len(segs), s, n, s, n, None, None, qkv.data_ptr(), 3 * D,
                                    qkv[:, D:].data_ptr(), 3 * D, vt.data_ptr(), ldv, o.data_ptr(), D, st))
    t2i.linear_i8(*t2i.quant_rows(o), *p["wo"], p["bo"], K=D, epilogue="resid", resid=resid)
    h = torch.empty_like(x)
    _lib.check(lib.t2i_op_ln_modulate(_lib.T2I_BF16, rows, D, resid.data_ptr(), p["mod"].data_ptr(),
                                      p["mod"][1].data_ptr(), 1e-6, h.data_ptr(), st))
    f, pre = t2i.gated_linear(h, p["wg"], p["wu"], p["bg"], p["bu"], act="gelu", save_pre=True)
    t2i.linear_i8(*t2i.quant_rows(f), *p["w2"], p["b2"], K=f.shape[1], epilogue="resid_gated", resid=resid,
                  gate=p["gate"])
    return resid, q, h, f, pre


def block_params(D, H, F):
    d = D // H
    p = dict(H=H, d=d)
    host = {}
    for i, (name, n, kk) in enumerate((("wqkv", 3 * D, D), ("wo", D, D), ("w2", D, F))):
        w, _ = rnd(200 + i, (n, kk), kk ** -0.5)
        p[name] = t2i.quant_rows(w)
        host[name] = (p[name][0].cpu().numpy()[:, :kk], p[name][1].cpu().numpy())
    for i, (name, shape, std, dt) in enumerate((
            ("bqkv", (3 * D,), 0.1, BF16), ("bo", (D,), 0.1, BF16), ("b2", (D,), 0.1, BF16),
            ("nq", (d,), 1.0, BF16), ("nk", (d,), 1.0, BF16), ("wg", (F, D), D ** -0.5, BF16),
            ("wu", (F, D), D ** -0.5, BF16), ("bg", (F,), 0.1, BF16), ("bu", (F,), 0.1, BF16),
            ("mod", (2, D), 0.3, F32), ("gate", (D,), 0.5, F32))):
        p[name], host[name] = rnd(300 + i, shape, std, dt)
    return p, host


def test_a_block_of_the_operators_together():
    D, H, F = 256, 4, 424
    segs = [(0, 77), (80, 130)]
    rows = 210
    p, h = block_params(D, H, F)
    x, hx = rnd(400, (rows, D), 1.0, BF16)
    resid, hr = rnd(401, (rows, D), 1.0)
    _, _, _, _, rot = qk_case(rows, H, H, D // H, BF16, "pairs", 17)
    out, q, hh, f, pre = chain(p, x, resid.clone(), rot, segs)

    # the same in float64, 8-bit rows where the block has them
    def lin(v, name, b):
        q8, s8 = blocks.quant_rows(v)
        return blocks.linear_i8(q8, s8, *h[name], h[b])
    qkv = lin(hx, "wqkv", "bqkv")
    hrot = host_rot(rot)
    q64 = blocks.qk_norm_rope(qkv[:, :D].reshape(rows, H, -1), h["nq"], 1e-6, **hrot).reshape(rows, D)
    k64 = blocks.qk_norm_rope(qkv[:, D:2 * D].reshape(rows, H, -1), h["nk"], 1e-6, **hrot).reshape(rows, D)
    o = np.zeros((rows, D))
    for a, n in segs:
        o[a:a + n] = dit.attention(q64[a:a + n], k64[a:a + n], qkv[a:a + n, 2 * D:], H)
    live = np.concatenate([np.arange(a, a + n) for a, n in segs])
    r1 = hr.copy()
    r1[live] += lin(o[live], "wo", "bo")
    mu = r1.mean(1, keepdims=True)
    ln = (r1 - mu) / np.sqrt(((r1 - mu) ** 2).mean(1, keepdims=True) + 1e-6) * (1 + h["mod"][1]) + h["mod"][0]
    g, u = blocks.gated_pre(ln, h["wg"], h["wu"], h["bg"], h["bu"])
    ref = r1 + h["gate"] * lin(blocks.gated("gelu", g, u), "w2", "b2")
    # every stage rounds its output to bf16 (at most 2^-8 of each value) and the
    # 8-bit rows differ where an input moves over a rounding border (a step of
    # 1 / 127 of the row's largest): eight stages of 2^-8 each
    assert rel_l2(to_host(q).reshape(rows, D)[live], q64[live]) < 3 * 2.0 ** -8
    assert rel_l2(to_host(out)[live], ref[live]) < 8 * 2.0 ** -8

    # the feed-forward's gradients with what the block kept
    dout, hd = rnd(402, (rows, F), 1.0, BF16)
    d = dict(x=hh, wg=p["wg"], wu=p["wu"])
    hst = dict(x=to_host(hh), wg=h["wg"], wu=h["wu"])
    check_backward(BF16, "gelu", d, hst, pre, dout, hd)


def test_on_another_stream_and_in_graphs():
    """The block on a side stream, and captured: every replay equals the eager result, with
    eager work between the replays; two graphs of the same calls do not share workspaces."""
    D, H, F, rows = 256, 4, 264, 130
    p, _ = block_params(D, H, F)
    x, _ = rnd(410, (rows, D), 1.0, BF16)
    resid, _ = rnd(411, (rows, D), 1.0)
    dout, _ = rnd(412, (rows, F), 1.0, BF16)
    _, _, _, _, rot = qk_case(rows, H, H, D // H, BF16, "halves", 19)
    dq, _ = rnd(413, (rows, H, D // H), 1.0, BF16)

    def work(r):
        r.copy_(resid)
        out, q, h, f, pre = chain(p, x, r, rot, [(0, rows)])
        g = t2i.gated_linear_backward(dout, h, p["wg"], p["wu"], pre, act="gelu", bias=True)
        b = t2i.qk_norm_rope_backward(dq, dq, q, q, p["nq"], p["nk"], **rot)
        return [out, f, *g, *b]

    eager = [t.clone() for t in work(torch.empty_like(resid))]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = work(torch.empty_like(resid))
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(a, b) for a, b in zip(eager, got))
    graphs = []
    for _ in range(2):
        r, g = torch.empty_like(resid), torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            out = work(r)
        graphs.append((g, out))
    for _ in range(3):
        for g, out in graphs:
            for t in out:
                t.fill_(3)
            g.replay()
            between = work(torch.empty_like(resid))
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(eager, out))
            assert all(torch.equal(a, b) for a, b in zip(eager, between))


def test_explicit_stream_argument():
    x, _ = rnd(420, (300, 256), 1.0, BF16)
    w, _ = rnd(421, (64, 256), 0.1, BF16)
    want = t2i.gated_linear(x, w, w)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    got = t2i.gated_linear(x, w, w, stream=s)
    s.synchronize()
    assert torch.equal(got, want)


@pytest.mark.parametrize("bad", [
    lambda x, q8, s8: t2i.quant_rows(x[:, ::2]), lambda x, q8, s8: t2i.quant_rows(x.half()),
    lambda x, q8, s8: t2i.quant_rows(x[:0]), lambda x, q8, s8: t2i.quant_rows(x[:1].expand(4, 256)),
    lambda x, q8, s8: t2i.quant_rows(x[0]),
    lambda x, q8, s8: t2i.linear_i8(q8, s8, q8, s8, K=257), lambda x, q8, s8: t2i.linear_i8(q8, s8[:3], q8, s8, K=256),
    lambda x, q8, s8: t2i.linear_i8(q8, s8, q8, s8, x[0], K=256), lambda x, q8, s8: t2i.linear_i8(x, s8, q8, s8, K=256),
    lambda x, q8, s8: t2i.linear_i8(q8, s8, q8, s8, K=256, epilogue="relu"),
    lambda x, q8, s8: t2i.linear_i8(q8, s8, q8, s8, K=256, epilogue="resid"),
    lambda x, q8, s8: t2i.linear_i8(q8, s8, q8, s8, K=256, resid=torch.zeros(8, 8, device=DEV)),
    lambda x, q8, s8: t2i.linear_i8(q8, s8, q8, s8, K=256, epilogue="resid_gated", resid=torch.zeros(8, 8, device=DEV)),
    lambda x, q8, s8: t2i.gated_linear(x, x, x[:4]), lambda x, q8, s8: t2i.gated_linear(x, x, x.float()),
    lambda x, q8, s8: t2i.gated_linear(x, x, x, act="relu"), lambda x, q8, s8: t2i.gated_linear(x, x, x, x[0, :8]),
    lambda x, q8, s8: t2i.gated_linear(x[:, :252], x[:, :252], x[:, :252]),
    lambda x, q8, s8: t2i.gated_linear(x[:, 1:249], x[:, 1:249], x[:, 1:249]),
    lambda x, q8, s8: t2i.gated_linear_backward(x[:, :8], x, x, x, x[:, :8]),
    lambda x, q8, s8: t2i.gated_linear_backward(x[:, :8], x, x, x, x[:, :16].float(), need_dx=False, need_dw=False),
    lambda x, q8, s8: t2i.gated_linear_backward(x[:, :8], x, x, x, x[:, :16]),
    lambda x, q8, s8: t2i.qk_norm_rope(x, x), lambda x, q8, s8: t2i.qk_norm_rope(x.view(8, 4, 64), x.view(8, 8, 32)),
    lambda x, q8, s8: t2i.qk_norm_rope(x.view(8, 4, 64), x.view(8, 4, 64).transpose(1, 2)),
    lambda x, q8, s8: t2i.qk_norm_rope(x.view(8, 4, 64), x.view(8, 4, 64), pos=torch.zeros(8, dtype=torch.int32, device=DEV)),
    lambda x, q8, s8: t2i.qk_norm_rope(x.view(8, 4, 64), x.view(8, 4, 64), table=torch.zeros(7, 32, 2, device=DEV)),
    lambda x, q8, s8: t2i.qk_norm_rope(x.view(8, 4, 64), x.view(8, 4, 64), table=torch.zeros(8, 64, device=DEV)),
    lambda x, q8, s8: t2i.qk_norm_rope(x.view(8, 4, 64), x.view(8, 4, 64), pairing="both"),
    lambda x, q8, s8: t2i.qk_norm_rope_backward(x.view(8, 4, 64), x.view(8, 4, 64), x.view(8, 4, 64), x.view(8, 4, 64)[:, :2]),
])
def test_python_calls_refuse(bad):
    x, _ = rnd(430, (8, 256), 1.0, BF16)
    with pytest.raises(t2i.T2IError):
        bad(x, *t2i.quant_rows(x))


# ------------------------------------------------------------------ forms that large inputs take

MANY_HEADS = [(1400, 24, 24, 128, "pairs"), (17000, 2, 1, 128, "halves"), (6000, 16, 5, 64, "halves"),
              (33000, 5, 1, 32, "pairs"), (4200, 4, 2, 256, "halves"), (14400, 1, 4, 72, "pairs"),
              (8400, 3, 4, 80, "halves"), (131100, 2, 1, 16, "halves"), (132000, 6, 1, 8, "pairs")]


@pytest.mark.parametrize("rows,hq,hk,d,pairing", MANY_HEADS)
@DTYPES
def test_qk_norm_rope_of_several_heads_per_group(rows, hq, hk, d, pairing, dtype):
    """Four heads of a row per group of lanes (backward: two), numbers of heads that they
    divide and that they do not, q and k within one group's heads."""
    say("qk, several heads", rows, hq, hk, d, pairing, NAME[dtype])
    heads = t2i.load().t2i_test_head_norm_heads
    assert heads(rows, hq + hk, d, 0) == 4 and heads(rows, hq + hk, d, 1) == 2
    q, k, wq, wk, rot = qk_case(rows, hq, hk, d, dtype, pairing, 21)
    dq, hdq = rnd(22, (rows, hq, d), 1.0, dtype)
    dk, hdk = rnd(23, (rows, hk, d), 1.0, dtype)
    eps, hr = 1e-3, host_rot(rot)
    out = t2i.qk_norm_rope(q, k, wq, wk, eps=eps, **rot)
    got = t2i.qk_norm_rope_backward(dq, dk, q, k, wq, wk, eps=eps, **rot)
    i = some(rows, 4)
    it, ri = torch.from_numpy(i).to(DEV), dict(hr, pos=hr["pos"][i])
    for x, w, dy, y, dx, dw in ((q, wq, hdq, out[0], got[0], got[2]), (k, wk, hdk, out[1], got[1], got[3])):
        hx, hw = to_host(x), to_host(w)
        # the bounds of the smaller cases' tests
        ref = blocks.qk_norm_rope(hx[i], hw, eps, **ri)
        mix = np.sqrt(pair_energy(blocks.head_norm(hx[i], hw, eps), pairing))
        tol = (d / 16 + 12) * E * 2 * np.maximum(mix, np.abs(ref))
        within(y[it], ref, tol + U[dtype] * (np.abs(ref) + tol))
        ref, _ = blocks.qk_norm_rope_grads(dy[i], hx[i], hw, eps, **ri)
        r = 1 / np.sqrt((hx * hx).mean(-1, keepdims=True) + eps)
        n, mix = hx * r, np.sqrt(pair_energy(dy, pairing))
        size = mix[i] * np.abs(hw)
        tol = 2 * (d / 16 + 16) * E * r[i] * (size + np.abs(n[i]) * (size * np.abs(n[i])).mean(-1, keepdims=True))
        within(dx[it], ref, tol + U[dtype] * (np.abs(ref) + tol), "dx")
        ref = (blocks.rotate(dy, hr["table"], hr["pos"], pairing, inverse=True) * n).sum((0, 1))
        # a term: rotation, root, product (d / 16 + 12 roundings); a lane's run of at most
        # rows heads / (1024 groups) terms, at least two heads per step; then wider sums
        tol = (rows * (hq + hk) / 1024 + 64 + d / 16) * E * (mix * np.abs(n)).sum((0, 1))
        within(dw, ref, tol + U[dtype] * (np.abs(ref) + tol), "dw")


@pytest.mark.parametrize("M,F,dtype,rows", [
    (333, 2048, BF16, 8), (1030, 2048, BF16, 16), (2101, 2048, BF16, 32), (4133, 2048, BF16, 64),
    (5001, 1608, BF16, 64), (301, 2055, F32, 8), (927, 2055, F32, 16), (1851, 2055, F32, 32), (3710, 2055, F32, 64)])
def test_bias_gradients_of_every_row_block(M, F, dtype, rows):
    """8 to 64 rows per workgroup, up to 8 of them per thread, a last block that is not full."""
    say("bias gradients", M, F, NAME[dtype], rows)
    assert t2i.load().t2i_test_gate_rows(M, F) == rows and M % rows
    d, _ = gated_case(M, F, 8, dtype, False, 170)
    pre, hp = rnd(171, (M, 2 * F), 1.5)
    dout, hd = rnd(172, (M, F), 1.0, dtype)
    got = t2i.gated_linear_backward(dout, d["x"], d["wg"], d["wu"], pre, act="gelu", bias=True, need_dx=False,
                                    need_dw=False)
    assert got[0] is None and got[1] is None and got[2] is None
    g, u = hp[:, :F], hp[:, F:]
    # per value as in the other gradients' tests; 8 rows in a thread, 8 threads, one
    # rounding of the block's sum, the rest wider
    for t, ref, each in ((got[3], hd * u * blocks.act_grad("gelu", g), np.abs(hd * u) * (1 + np.abs(g))),
                         (got[4], hd * blocks.act("gelu", g), np.abs(hd * g))):
        f = 2.0 ** -20 * each
        tol = f.sum(0) + 17 * E * (np.abs(ref) + f).sum(0)
        ref = ref.sum(0)
        within(t, ref, tol + U[dtype] * (np.abs(ref) + tol))


@pytest.mark.parametrize("M,N,K", [(1, 70, 300), (5, 128, 128), (33, 3000, 650), (70, 1152, 1152), (300, 260, 700),
                                   (200, 1033, 650), (2050, 1152, 256), (4090, 4090, 640)])
def test_linear_i8_residual_updates_with_fp32_biases(M, N, K):
    a, sa, w, sw = i8_operands(M, N, K, 3)
    d = [dev(v, torch.int8) if v.dtype == np.int8 else dev(v) for v in (a, sa, w, sw)]
    b, rb = rnd(10, (N,), 0.3, F32)
    gate, rg = rnd(11, (N,), 0.5)
    x0, rx = rnd(12, (M, N), 2.0)
    i = some(M, 5)
    it = torch.from_numpy(i).to(DEV)
    y = (a[i, :K].astype(np.float64) @ w[:, :K].astype(np.float64).T) * sa[i, None].astype(np.float64) * sw + rb
    for epi, g in (("resid", np.ones(N)), ("resid_gated", rg)):
        x, buf = padded(x0, 3)
        cp, cbuf = padded(x0.to(BF16), 3)
        out = t2i.linear_i8(*d, b, K=K, epilogue=epi, dtype=F32, resid=x, resid_copy=cp,
                            gate=gate if epi == "resid_gated" else None)
        assert out is x
        ref = rx[i] + g * y
        tol = np.abs(g) * i8_bound(y - rb, rb, y, F32, "store") + 2 * E * (np.abs(g * y) + np.abs(ref))
        within(x[it], ref, tol, epi)
        assert torch.equal(cp, x.to(BF16)) and (cbuf[:-1, N:] == 7).all()
        assert (buf[:-1, N:] == 7).all() and (buf[-1] == 7).all()


# ------------------------------------------------------------------ sums that cancel

@pytest.mark.parametrize("d", [8, 64, 72, 128])
@DTYPES
def test_head_weight_gradients_that_cancel(d, dtype):
    """One head per group: 2^24, ones, -2^24.  In fp32 the groups' sum loses every one."""
    groups = {8: 256, 64: 32, 72: 28, 128: 16}[d]
    one = torch.ones((groups, 1, d), dtype=dtype, device=DEV)
    dy = one.clone()
    dy[0], dy[-1] = 2.0 ** 24, -2.0 ** 24
    w = torch.ones(d, dtype=dtype, device=DEV)
    # (mean 1, eps 0: every normed value is the root's reciprocal, the same for all)
    norm = t2i.qk_norm_rope(one, one[:, :0], w, w, eps=0.0)[0][0, 0].double()
    dw = t2i.qk_norm_rope_backward(dy, one[:, :0], one, one[:, :0], w, w, eps=0.0)[2].double()
    want = (groups - 2) * norm
    assert ((dw - want).abs() <= 2 * U[dtype] * want).all(), dw


@DTYPES
def test_bias_gradients_that_cancel(dtype):
    """One row per thread: 2^24, ones, -2^24, times an activation of 64 (exact)."""
    M, F = 8, 16
    dout = torch.ones((M, F), dtype=dtype, device=DEV)
    dout[0], dout[-1] = 2.0 ** 24, -2.0 ** 24
    x, w = torch.ones((M, 8), dtype=dtype, device=DEV), torch.ones((F, 8), dtype=dtype, device=DEV)
    pre = torch.full((M, 2 * F), 64.0, device=DEV)
    for act in ("silu", "gelu"):
        dbu = t2i.gated_linear_backward(dout, x, w, w, pre, act=act, bias=True)[4]
        assert (dbu == 64.0 * (M - 2)).all(), (act, dbu)


# ------------------------------------------------------------------ beside automatic differentiation

class Gated(torch.autograd.Function):
    """The gated block as a program would record it: the calls in passes that record nothing."""

    @staticmethod
    def forward(ctx, x, wg, wu):
        out, pre = t2i.gated_linear(x, wg, wu, act="gelu", save_pre=True)
        ctx.save_for_backward(x, wg, wu, pre)
        return out

    @staticmethod
    def backward(ctx, dout):
        return t2i.gated_linear_backward(dout, *ctx.saved_tensors, act="gelu")[:3]


def test_calls_inside_an_autograd_function():
    d, _ = gated_case(70, 72, 136, BF16, False, 180)
    dout, _ = rnd(181, (70, 72), 1.0, BF16)
    out, pre = t2i.gated_linear(d["x"], d["wg"], d["wu"], act="gelu", save_pre=True)
    want = t2i.gated_linear_backward(dout, d["x"], d["wg"], d["wu"], pre, act="gelu")[:3]
    leaves = [d[n].clone().requires_grad_() for n in ("x", "wg", "wu")]
    with pytest.raises(t2i.T2IError):
        t2i.gated_linear(*leaves, act="gelu")
    y = Gated.apply(*leaves)
    assert torch.equal(y, out)
    y.backward(dout)
    assert all(torch.equal(t.grad, g) for t, g in zip(leaves, want))
    with torch.no_grad():
        assert torch.equal(t2i.gated_linear(*leaves, act="gelu"), out)


def test_a_saved_operand_overwritten_in_place_is_found():
    q, k, wq, wk, rot = qk_case(37, 4, 2, 64, F32, "halves", 24, fused=False)
    weight = torch.ones_like(q).requires_grad_()
    y = (weight * q).sum()
    t2i.qk_norm_rope(q, k, wq, wk, inplace=True, **rot)
    with pytest.raises(RuntimeError, match="inplace"):
        y.backward()
