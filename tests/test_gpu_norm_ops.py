"""The residual's addition with an RMS norm, its 8-bit form and its gradients on the GPU
against their float64 definitions (``oracle/blocks.py``).

Bounds count roundings, U half a step of the result's type relative to the value, E =
2^-24.  A row's sum takes at most 32 values in a chain, then at most 24 more additions (16
waves or lanes in twos), so that the sum of squares is off by at most 56 E of itself and r
= (.)^-1/2 by half of that and its own 2 E; with the two products of y 40 E are never
reached.  A sum with signs is off by 56 E of the sum of sizes."""
import ctypes as C

import numpy as np
import pytest
import torch

import paper_2607_26566_amd as t2i
from paper_2607_26566_amd import _lib
from oracle import blocks
from gpu_common import DEV, say, to_host
from test_gpu_block_ops import BF16, DTYPES, E, F32, NAME, U, dev, padded, rnd, within

pytestmark = pytest.mark.gpu
EPS = 1e-5

# every number of pieces per thread and of threads per row, rows of one element and of
# several rounds, widths off eight
SIZES = [(1, 1), (3, 7), (5, 8), (9, 64), (2, 511), (4, 512), (3, 513), (6, 1051), (70, 1152), (5, 1537), (2, 2047),
         (3, 2049), (2, 4096), (3, 4097), (2, 8193), (2, 12289), (3, 16384), (2, 16385), (2, 40003)]
# (operands' type, residual's type or None)
TYPES = [(BF16, None), (BF16, BF16), (BF16, F32), (F32, None), (F32, F32)]
TYPED = pytest.mark.parametrize("dtype,rtype", TYPES, ids=lambda t: "none" if t is None else NAME[t])


def operands(rows, K, dtype, rtype, seed=0):
    x, _ = rnd(seed + rows * 7 + K, (rows, K), 1.0, dtype)
    w, _ = rnd(seed + K + 1, (K,), 0.3, dtype)
    resid = None if rtype is None else rnd(seed + rows + K + 2, (rows, K), 2.0, rtype)[0]
    h = x if resid is None else (resid.float() + x.float()).to(rtype)
    return x, w + 1, resid, h


@pytest.mark.parametrize("rows,K", SIZES)
@TYPED
def test_add_rms_norm(rows, K, dtype, rtype):
    say("norm", rows, K, NAME[dtype], rtype)
    x, w, resid, h = operands(rows, K, dtype, rtype)
    for weight in (w, None):
        y, got = t2i.add_rms_norm(x, weight, resid, eps=EPS)
        assert (got is x) if resid is None else (got.dtype == rtype and torch.equal(got, h))
        assert y.dtype == dtype
        ref = blocks.add_rms_norm(to_host(h), None if weight is None else to_host(w), EPS)
        within(y, ref, (U[dtype] + 40 * E) * np.abs(ref) + 40 * E * U[dtype] * np.abs(ref), weight is None)


@pytest.mark.parametrize("rows,K", SIZES)
@TYPED
def test_add_rms_norm_i8(rows, K, dtype, rtype):
    say("norm i8", rows, K, NAME[dtype], rtype)
    x, w, resid, h = operands(rows, K, dtype, rtype, 5)
    for weight in (w, None):
        q, s, got = t2i.add_rms_norm_i8(x, weight, resid, eps=EPS)
        assert (got is x) if resid is None else torch.equal(got, h)
        rq, rs = blocks.add_rms_norm_i8(to_host(h), None if weight is None else to_host(w), EPS)
        q = q.cpu().numpy()
        assert q.shape == (rows, (K + 127) // 128 * 128)
        assert np.array_equal(q[:, :K], rq) and not q[:, K:].any()
        # r, its product with T and the division by 127
        within(s, rs, 42 * E * rs)


@TYPED
def test_codes_at_halves_and_beside_them(dtype, rtype):
    """Quotients that lie at a half, and the values next to them, at several sizes; the last rows
    need products past fp32's range or lose bits there."""
    half = np.arange(-127, 127) + 0.5
    rows = []
    for top in (127.0, 254.0, 3.0, 0.7, 2.0 ** -60, 2.0 ** 100, 2.0 ** -110, 2.0 ** 121):
        near = dev((half * (top / 127)).astype(np.float32), dtype)
        for v in (near, torch.nextafter(near, torch.full_like(near, 3e38)), torch.nextafter(near, -torch.full_like(near, 3e38))):
            rows.append(np.concatenate([np.clip(to_host(v), -top, top), [top, 0.5 * top, -0.5 * top, 0]]))
    h = dev(np.stack(rows).astype(np.float32), dtype)
    K = h.shape[1]
    # weights that are powers of two keep the halves; others move them
    for w in (None, dev(2.0 ** np.random.default_rng(1).integers(-2, 1, K), dtype), dev(np.full(K, 0.7), dtype),
              rnd(3, (K,), 1.0, dtype)[0]):
        x, resid = (h, None) if rtype is None else (torch.zeros_like(h), h.to(rtype))
        q, s, _ = t2i.add_rms_norm_i8(x, w, resid, eps=0.0)
        rq, rs = blocks.add_rms_norm_i8(to_host(h), None if w is None else to_host(w), 0.0)
        assert np.array_equal(q.cpu().numpy()[:, :K], rq)
        size = np.abs(to_host(h)).max(1)
        usual = (size > 1e-17) & (size < 1e17)    # squares within fp32
        within(s[torch.from_numpy(usual).to(DEV)], rs[usual], 42 * E * rs[usual])


@TYPED
def test_rows_that_are_not_finite_or_zero_stay_apart(dtype, rtype):
    rows, K = 9, 2100
    x, w, resid, _ = operands(rows, K, dtype, rtype, 9)
    at = x if resid is None else resid
    at[1, 3], at[3, 2099], at[5, 0] = float("nan"), float("inf"), float("-inf")
    x[7] = 0
    if resid is not None:
        resid[7] = 0
    h = x if resid is None else (resid.float() + x.float()).to(rtype)
    good = [0, 2, 4, 6, 8]
    y, got = t2i.add_rms_norm(x, w, resid, eps=EPS)
    assert torch.equal(got.nan_to_num(7, 7, 7), h.nan_to_num(7, 7, 7))
    alone, _ = t2i.add_rms_norm(x[good], w, None if resid is None else resid[good], eps=EPS)
    assert torch.equal(y[good], alone) and not y[7].any()
    assert y[[1, 3, 5]].isnan().any(1).all()
    q, s, _ = t2i.add_rms_norm_i8(x, w, resid, eps=EPS)
    rq, rs = blocks.add_rms_norm_i8(to_host(h), to_host(w), EPS)
    assert np.array_equal(q.cpu().numpy()[:, :K], rq)
    assert s[[1, 3, 5]].isnan().all() and not q[[1, 3, 5, 7]].any() and s[7] == 0
    # a row of zeros with eps 0: 0 / 0
    assert t2i.add_rms_norm(x[7:8], w, None if resid is None else resid[7:8], eps=0.0)[0].isnan().all()
    # squares past fp32
    big = torch.full((1, 40), 1e30, dtype=dtype, device=DEV)
    assert not t2i.add_rms_norm(big, eps=EPS)[0].any()
    # products past fp32 in one row only
    h2 = torch.ones((2, 40), dtype=dtype, device=DEV)
    h2[0] = 1e20
    q, s, _ = t2i.add_rms_norm_i8(h2, torch.full((40,), 1e20, dtype=dtype, device=DEV))
    assert s[0].isnan() and not q[0].any() and s[1].isfinite() and (q[1, :40] == 127).all()


@TYPED
def test_norm_strides_surroundings_and_in_place(dtype, rtype):
    lib, st = t2i.load(), C.c_void_p(torch.cuda.current_stream().cuda_stream)
    for rows, K in ((5, 300), (3, 2051), (2, 16500)):
        x, w, resid, h = operands(rows, K, dtype, rtype, 13)
        y0, _ = t2i.add_rms_norm(x, w, resid, eps=EPS)
        q0, s0, _ = t2i.add_rms_norm_i8(x, w, resid, eps=EPS)
        for extra in (1, 8):
            xs, _ = padded(x, extra)
            wide = torch.full((K + 1,), 9.0, dtype=dtype, device=DEV)   # (a weight off 16 bytes)
            wide[1:] = w
            rs = None if resid is None else padded(resid, extra + 2)[0]
            y, g = t2i.add_rms_norm(xs, wide[1:], rs, eps=EPS)
            assert torch.equal(y, y0) and torch.equal(g, h)
            q, s, _ = t2i.add_rms_norm_i8(xs, wide[1:], rs, eps=EPS)
            assert torch.equal(q, q0) and torch.equal(s, s0)
            # outputs inside larger buffers, y over x
            hb = None if resid is None else padded(h * 0, extra)
            _lib.check(lib.t2i_op_add_rms_norm(
                int(dtype == BF16), int((rtype or dtype) == BF16), rows, K, xs.data_ptr(), xs.stride(0),
                None if rs is None else rs.data_ptr(), K if rs is None else rs.stride(0), w.data_ptr(), EPS,
                None if hb is None else hb[0].data_ptr(), K if hb is None else hb[0].stride(0), xs.data_ptr(),
                xs.stride(0), st))
            assert torch.equal(xs, y0)
            whole = xs.as_strided((rows + 1, K + extra), (K + extra, 1))
            assert (whole[:rows, K:] == 7).all() and (whole[rows] == 7).all()
            if hb is not None:
                assert torch.equal(hb[0], h) and (hb[1][:-1, K:] == 7).all() and (hb[1][-1] == 7).all()
            ldq = (K + 127) // 128 * 128 + 16
            qb, sb = torch.full((rows + 1, ldq), 99, dtype=torch.int8, device=DEV), torch.full((rows + 1,), 5.0, device=DEV)
            xs.copy_(x)
            _lib.check(lib.t2i_op_add_rms_norm_i8(
                int(dtype == BF16), int((rtype or dtype) == BF16), rows, K, xs.data_ptr(), xs.stride(0),
                None if rs is None else rs.data_ptr(), K if rs is None else rs.stride(0), w.data_ptr(), EPS,
                None if hb is None else hb[0].data_ptr(), K if hb is None else hb[0].stride(0), qb.data_ptr(), ldq,
                sb.data_ptr(), st))
            assert torch.equal(qb[:rows, :-16], q0) and (qb[:rows, -16:] == 99).all() and (qb[rows] == 99).all()
            assert torch.equal(sb[:rows], s0) and sb[rows] == 5
            if resid is not None:
                for call in (t2i.add_rms_norm, t2i.add_rms_norm_i8):
                    rs, buf = padded(resid, extra)
                    before = rs._version
                    out = call(x, w, rs, eps=EPS, inplace=True)
                    assert out[-1] is rs and torch.equal(rs, h) and rs._version == before + 1
                    assert torch.equal(out[0], y0 if call is t2i.add_rms_norm else q0)
                    assert (buf[:-1, K:] == 7).all() and (buf[-1] == 7).all()


@pytest.mark.parametrize("K", [513, 1051, 1152, 2048, 3001, 4096, 8192, 10007])
def test_norm_rows_do_not_depend_on_the_number_of_rows(K):
    """few rows have more threads each, and the same sums"""
    say("few and many rows", K)
    x, _ = rnd(81, (2100, K), 1.0, BF16)
    resid, _ = rnd(82, (2100, K), 2.0, F32)
    w, _ = rnd(83, (K,), 1.0, BF16)
    y, h = t2i.add_rms_norm(x, w, resid, eps=EPS)
    q, s, _ = t2i.add_rms_norm_i8(x, w, resid, eps=EPS)
    for rows in (1, 200, 300, 1024, 2048):
        fy, fh = t2i.add_rms_norm(x[:rows], w, resid[:rows], eps=EPS)
        fq, fs, _ = t2i.add_rms_norm_i8(x[:rows], w, resid[:rows], eps=EPS)
        assert torch.equal(fy, y[:rows]) and torch.equal(fh, h[:rows])
        assert torch.equal(fq, q[:rows]) and torch.equal(fs, s[:rows])


def test_norm_rows_do_not_depend_on_the_batch():
    x, w, resid, _ = operands(3000, 1152, BF16, F32, 17)
    y, _ = t2i.add_rms_norm(x, w, resid)
    q, s, _ = t2i.add_rms_norm_i8(x, w, resid)
    for a, b in ((0, 1), (17, 20), (1000, 2999)):
        assert torch.equal(t2i.add_rms_norm(x[a:b], w, resid[a:b])[0], y[a:b])
        qb, sb, _ = t2i.add_rms_norm_i8(x[a:b], w, resid[a:b])
        assert torch.equal(qb, q[a:b]) and torch.equal(sb, s[a:b])


# ------------------------------------------------------------------ gradients

def grad_operands(rows, K, dtype, rtype, seed=0):
    h, _ = rnd(seed + rows * 3 + K, (rows, K), 2.0, rtype or dtype)
    return (rnd(seed + K + 1, (rows, K), 1.0, dtype)[0], h, rnd(seed + K + 2, (K,), 0.3, dtype)[0] + 1,
            rnd(seed + rows + 3, (rows, K), 1.0, rtype or dtype)[0])


def grad_bounds(dy, h, w, dh, dtype, rtype, chain=64):
    """(dsum, dw and the bounds of both) in float64"""
    dy, h, dh = to_host(dy), to_host(h), None if dh is None else to_host(dh)
    w = None if w is None else to_host(w)
    ds, dw = blocks.add_rms_norm_grads(dy, h, w, dh, EPS)
    r = 1 / np.sqrt((h * h).mean(-1, keepdims=True) + EPS)
    n, d = np.abs(h * r), np.abs(dy if w is None else dy * w)
    # mean(d n): 56 E of the sizes' mean and r's error; four products and sums of each term
    err = 100 * E * r * (d + n * (d * n).mean(-1, keepdims=True)) + 2 * E * (0 if dh is None else np.abs(dh))
    # a workgroup's rows in a chain of `chain`, the rest in float64; r, the products, the sum kept in fp32
    return ds, err, dw, (chain + 34) * E * (np.abs(dy) * n).sum(0)


@pytest.mark.parametrize("rows,K", SIZES + [(300, 1152), (3001, 72), (2200, 2056), (1300, 4104), (1100, 9000)])
@pytest.mark.parametrize("dtype,rtype", [(BF16, BF16), (BF16, F32), (F32, F32)], ids=NAME.get)
def test_add_rms_norm_backward(rows, K, dtype, rtype):
    say("norm bwd", rows, K, NAME[dtype], NAME[rtype])
    dy, h, w, dh = grad_operands(rows, K, dtype, rtype)
    for weight, other in ((w, dh), (w, None), (None, dh)):
        dx, dresid, dw = t2i.add_rms_norm_backward(dy, h, weight, other, eps=EPS)
        ds, err, rdw, werr = grad_bounds(dy, h, weight, other, dtype, rtype)
        within(dx, ds, U[dtype] * (np.abs(ds) + err) + err, "dx")
        assert dx.dtype == dtype
        if rtype == dtype:
            assert dresid is None
        else:
            assert dresid.dtype == rtype and torch.equal(dresid.to(dtype), dx)
            within(dresid, ds, U[rtype] * np.abs(ds) + err, "dresid")
        if weight is None:
            assert dw is None
        else:
            within(dw, rdw, U[dtype] * (np.abs(rdw) + werr) + werr, "dw")


def test_norm_weight_gradients_that_cancel():
    """Rows in pairs whose terms cancel but for a small rest: chains of fp32 sums lose little of it."""
    rows, K = 40000, 64
    dy, h, w, _ = grad_operands(rows, K, F32, F32, 21)
    h[1::2] = -h[0::2]
    dy[1::2] = dy[0::2] * (1 + 2.0 ** -10)
    _, _, dw = t2i.add_rms_norm_backward(dy, h, w, eps=EPS)
    _, _, rdw, werr = grad_bounds(dy, h, w, None, F32, F32)
    within(dw, rdw, E * np.abs(rdw) + werr)


@pytest.mark.parametrize("dtype,rtype", [(BF16, BF16), (BF16, F32), (F32, F32)], ids=NAME.get)
def test_norm_backward_strides_in_place_and_rows_not_finite(dtype, rtype):
    lib, st = t2i.load(), C.c_void_p(torch.cuda.current_stream().cuda_stream)
    for rows, K in ((7, 300), (5, 2051), (3, 16384)):
        dy, h, w, dh = grad_operands(rows, K, dtype, rtype, 31)
        dx0, dr0, dw0 = t2i.add_rms_norm_backward(dy, h, w, dh, eps=EPS)
        for extra in (1, 8):
            s = [padded(t, extra)[0] for t in (dy, h, dh)]
            dx, dr, dw = t2i.add_rms_norm_backward(s[0], s[1], w, s[2], eps=EPS)
            assert torch.equal(dx, dx0) and torch.equal(dw, dw0) and (dr is None or torch.equal(dr, dr0))
            # dx over dy, dresid over dh
            n = lib.t2i_op_add_rms_norm_backward_ws_bytes(rows, K)
            ws = torch.full((n,), 0xff, dtype=torch.uint8, device=DEV)
            dw = torch.empty_like(w)
            _lib.check(lib.t2i_op_add_rms_norm_backward(
                int(dtype == BF16), int(rtype == BF16), rows, K, s[0].data_ptr(), s[0].stride(0), s[1].data_ptr(),
                s[1].stride(0), w.data_ptr(), EPS, s[2].data_ptr(), s[2].stride(0), s[0].data_ptr(), s[0].stride(0),
                s[2].data_ptr(), s[2].stride(0), dw.data_ptr(), ws.data_ptr(), n, st))
            assert torch.equal(s[0], dx0) and torch.equal(dw, dw0)
            assert torch.equal(s[2], dx0 if dr0 is None else dr0)
            for t in s:
                whole = t.as_strided((rows + 1, K + extra), (K + extra, 1))
                assert (whole[:rows, K:] == 7).all() and (whole[rows] == 7).all()
        bad = h.clone()
        bad[1, 5] = float("nan")
        dx, _, dw = t2i.add_rms_norm_backward(dy, bad, w, dh, eps=EPS)
        keep = [i for i in range(rows) if i != 1]
        assert torch.equal(dx[keep], dx0[keep]) and dx[1].isnan().all() and dw.isnan().all()


def test_norm_on_another_stream_and_in_graphs():
    """Captured calls, replayed with eager work between, and the two directions as they follow each
    other."""
    x, w, resid, _ = operands(700, 1152, BF16, F32, 41)
    dy, dh = rnd(42, (700, 1152), 1.0, BF16)[0], rnd(43, (700, 1152), 1.0, F32)[0]

    def work():
        y, h = t2i.add_rms_norm(x, w, resid)
        q, s, _ = t2i.add_rms_norm_i8(x, w, resid)
        return (y, h, q, s, *t2i.add_rms_norm_backward(dy, h, w, dh))
    ref = [t.clone() for t in work()]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    y, _ = t2i.add_rms_norm(x, w, resid, stream=side)
    side.synchronize()
    assert torch.equal(y, ref[0])
    with torch.cuda.stream(side):
        work()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = work()
    for i in range(4):
        for t in out:
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(out, ref):
            assert torch.equal(a, b)
        dx = t2i.add_rms_norm_backward(dy, ref[1], w, dh)[0]
        assert torch.equal(dx, ref[4])
        if i == 1:     # new inputs in the same place
            x.copy_(x.flip(0))
            ref = [t.clone() for t in work()]


@pytest.mark.parametrize("bad", ["w", "resid_dtype", "resid_shape", "x_dim", "columns", "inplace", "dh", "host", "eps",
                                 "grad"])
def test_python_norm_calls_refuse(bad):
    x, w, resid, _ = operands(4, 64, BF16, F32)
    fwd = dict(x=x, w=w, resid=resid)
    kw = {}
    if bad == "w":
        fwd["w"] = w.float()
    elif bad == "resid_dtype":
        fwd.update(x=x.float(), w=w.float(), resid=x)
    elif bad == "resid_shape":
        fwd["resid"] = resid[:3]
    elif bad == "x_dim":
        fwd["x"] = x[0]
    elif bad == "columns":
        fwd["x"] = x.T.contiguous().T
    elif bad == "inplace":
        fwd["resid"], kw["inplace"] = None, True
    elif bad == "host":
        fwd["w"] = w.cpu()
    elif bad == "eps":
        kw["eps"] = -1.0
    elif bad == "grad":
        fwd["w"] = w.requires_grad_()
    for call in (t2i.add_rms_norm, t2i.add_rms_norm_i8):
        if bad != "dh":
            with pytest.raises(t2i.T2IError):
                call(**fwd, **kw)
    dy, h, w, dh = grad_operands(4, 64, BF16, F32)
    t2i.add_rms_norm_backward(dy, h, w, dh)
    with pytest.raises(t2i.T2IError):
        t2i.add_rms_norm_backward(dy, h, w, dh.to(BF16))
    with pytest.raises(t2i.T2IError):
        t2i.add_rms_norm_backward(dy.float(), h.to(BF16), w.float(), dh.to(BF16))
