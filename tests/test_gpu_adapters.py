"""Adapters of many requests beside a shared linear layer on the GPU against their float64
definitions (``oracle/blocks.py``).

Bounds count roundings.  U is half a step of the operands' type relative to the value, E =
2^-24; a sum of n products in fp32 is off by at most n E times the sum of the products'
sizes.  t (and the gradients' u) is such a sum, scaled, in fp32; the products take bf16
operands' as two bf16 values, 2^-16 of it short.  What it is off by goes through them."""
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
A = np.abs


def indexes(order, M, n, seed=0):
    """None, or the rows' adapters: requests one after the other, or every row for itself; some
    without (negative, or past the last)."""
    r = np.random.default_rng(seed + M)
    if order is None:
        return None
    if order == "scattered":
        return r.integers(-1, n + 1, M)
    if order == "one":
        return np.full(M, n - 1)
    ends = np.sort(r.integers(0, M + 1, 2 * n))
    return r.permutation(np.r_[np.arange(n), np.arange(n), [-1]])[np.searchsorted(ends, np.arange(M), side="right")]


def operands(M, N, K, n, rank, order, dtype, seed=0, scaled=True):
    s = seed + M * 5 + N * 3 + K + rank
    o = dict(x=rnd(s, (M, K), 1.0, dtype)[0], w=rnd(s + 1, (N, K), K ** -0.5, dtype)[0],
             a=rnd(s + 2, (n, rank, K), K ** -0.5, dtype)[0], b=rnd(s + 3, (n, N, rank), 0.5 * rank ** -0.5, dtype)[0])
    scale = dev(np.random.default_rng(s).uniform(0.5, 2, n)) if scaled else None
    ix = indexes(order, M, n, seed)
    index = None if ix is None else torch.from_numpy(ix.astype(np.int32)).to(DEV)
    return o, dict(index=index, scale=scale)


def host(o, kw):
    h = {k: to_host(v) for k, v in o.items()}
    h.update(index=None if kw["index"] is None else kw["index"].cpu().numpy(),
             scale=None if kw["scale"] is None else to_host(kw["scale"]))
    return h


def forward_bounds(h, bias, dtype):
    """(y, what it is off by before its own rounding, t, what t is off by)"""
    y, t = blocks.adapter_linear(**h, bias=bias)
    mag = {**h, **{k: A(h[k]) for k in "xwab"}}
    _, tm = blocks.adapter_linear(**mag)
    t_err = (h["x"].shape[1] + 2) * E * tm
    left = t_err + (2.0 ** -16 * A(t) if dtype == BF16 else 0)   # as the products take it
    K, rank = h["x"].shape[1], h["a"].shape[1]
    err = (K + 2) * E * (A(h["x"]) @ A(h["w"]).T) + 4 * E * A(y) + (0 if bias is None else 2 * E * A(bias))
    for i, rows in enumerate(blocks.adapter_rows(h["index"], h["a"].shape[0], y.shape[0])):
        err[rows] += (left[rows] + (2 * rank + 2) * E * A(t[rows])) @ A(h["b"][i]).T
    return y, err, t, t_err


# every kind of the narrow product (up to 64 rows, more), ranks on and off whole pieces, up to the largest, and
# tiles of 16 to 256 rows
SHAPES = [(1, 8, 8, 1, 1), (1, 4096, 1152, 1, 16), (2, 72, 136, 3, 5), (5, 128, 64, 2, 8), (16, 96, 504, 4, 4),
          (24, 4096, 520, 16, 16), (33, 1152, 96, 5, 33), (63, 64, 64, 3, 128), (64, 2304, 1000, 8, 3),
          (65, 136, 136, 2, 7), (100, 1000, 1152, 40, 8), (127, 1000, 1152, 4, 17), (257, 304, 1152, 6, 64),
          (333, 1152, 2056, 3, 16), (520, 2304, 384, 12, 100), (1025, 776, 136, 8, 32), (2100, 4608, 1152, 8, 12),
          (4000, 4096, 640, 5, 40), (3600, 3328, 776, 5, 16), (4000, 2816, 776, 7, 8), (4600, 1152, 2056, 3, 16),
          (3600, 640, 4104, 4, 24)]


# (fp32 takes the same tiles for more rows as for fewer)
CASES = pytest.mark.parametrize("M,N,K,n,rank,dtype", [(*s, d) for s in SHAPES for d in (BF16, F32)
                                                       if s[0] <= 1500 or d == BF16])
ORDERS = pytest.mark.parametrize("order", [None, "runs", "scattered", "one"])


@ORDERS
@CASES
def test_adapter_linear(M, N, K, n, rank, order, dtype):
    n = 1 if order is None else n
    say("adapter", M, N, K, n, rank, order, NAME[dtype])
    o, kw = operands(M, N, K, n, rank, order, dtype)
    bias, hb = rnd(9, (N,), 0.3, dtype)
    y, err, t, t_err = forward_bounds(host(o, kw), hb, dtype)
    out, got = t2i.adapter_linear(**o, bias=bias, **kw, save_t=True)
    assert out.dtype == dtype and got.shape == (M, (rank + 31) // 32 * 32) and not got[:, rank:].any()
    within(got[:, :rank], t, t_err, "t")
    within(out, y, U[dtype] * (A(y) + err) + err, "y")


@pytest.mark.parametrize("order", [None, "runs", "scattered"])
@pytest.mark.parametrize("K,rank", [(72, 9), (520, 16), (520, 20), (523, 50), (264, 100)])
@DTYPES
def test_narrow_products_of_more_tiles_than_cus(K, rank, order, dtype):
    """More than 4096 rows, with the gradients of both kinds."""
    M, N = 4200, 64
    if dtype == BF16:
        K = K // 8 * 8
    o, kw = operands(M, N, K, 1 if order is None else 5, rank, order, dtype, 23)
    h = host(o, kw)
    y, err, t, t_err = forward_bounds(h, None, dtype)
    out, got = t2i.adapter_linear(**o, **kw, save_t=True)
    within(got[:, :rank], t, t_err, "t")
    assert not got[:, rank:].any()
    within(out, y, U[dtype] * (A(y) + err) + err, "y")
    dy, hdy = rnd(24, (M, N), 1.0, dtype)
    grads = t2i.adapter_linear_backward(dy, **o, t=got, **kw)
    ref, bounds = backward_bounds(h, hdy, dtype)
    for v, name in zip(grads, ("dx", "da", "db")):
        within(v, ref[name], U[dtype] * (A(ref[name]) + bounds[name]) + bounds[name], name)


def check_all(o, kw, M, N, dtype, seed):
    h = host(o, kw)
    y, err, t, t_err = forward_bounds(h, None, dtype)
    out, got = t2i.adapter_linear(**o, **kw, save_t=True)
    within(got[:, :t.shape[1]], t, t_err, "t")
    within(out, y, U[dtype] * (A(y) + err) + err, "y")
    dy, hdy = rnd(seed, (M, N), 1.0, dtype)
    ref, bounds = backward_bounds(h, hdy, dtype)
    for v, name in zip(t2i.adapter_linear_backward(dy, **o, t=got, **kw), ("dx", "da", "db")):
        within(v, ref[name], U[dtype] * (A(ref[name]) + bounds[name]) + bounds[name], name)


@pytest.mark.parametrize("M,n", [(300, 1), (300, 2), (300, 4), (300, 300), (700, 512), (700, 600), (4100, 30), (8200, 3)])
@DTYPES
def test_rows_of_many_adapters(M, n, dtype):
    """Rows shared anew between tiles (more than three adapters to a tile, up to 512 in all), in one
    window and in two, and the other ways."""
    N, K = 16, 520
    o, kw = operands(M, N, K, n, 8, "scattered", dtype, 25)
    check_all(o, kw, M, N, dtype, 26)
    # single tiles of several adapters among tiles of one
    kw["index"] = torch.arange(M, device=DEV, dtype=torch.int32) // 48 % n
    kw["index"][33:61] = torch.arange(28, device=DEV, dtype=torch.int32) % n
    kw["index"][M - 9:] = torch.arange(9, device=DEV, dtype=torch.int32) % n
    check_all(o, kw, M, N, dtype, 27)


def test_rows_of_many_adapters_far_apart():
    """Rows of x that a window's 32-bit offsets do not reach."""
    M, N, K, ld = 300, 64, 72, 2 ** 18 + 8
    o, kw = operands(M, N, K, 9, 8, "scattered", BF16, 29)
    wide = torch.zeros((M - 1) * ld + K, dtype=BF16, device=DEV).as_strided((M, K), (ld, 1))
    wide.copy_(o["x"])
    y, t = t2i.adapter_linear(**o, **kw, save_t=True)
    y2, t2 = t2i.adapter_linear(**{**o, "x": wide}, **kw, save_t=True)
    assert torch.equal(t, t2) and torch.equal(y, y2)


@pytest.mark.parametrize("M,N,K,rank", [(1, 4096, 456, 16), (16, 4096, 1160, 9), (17, 2048, 520, 33), (17, 2056, 520, 8),
                                        (64, 1000, 456, 128), (64, 1032, 448, 16), (250, 256, 2056, 4), (15, 8, 5000, 1)])
def test_few_tiles_of_the_second_product(M, N, K, rank):
    """Up to one 16 x 16 tile to a CU, and a few more; groups of waves with a step and more each."""
    for order in (None, "runs", "scattered"):
        o, kw = operands(M, N, K, 1 if order is None else 4, rank, order, BF16, 31)
        check_all(o, kw, M, N, BF16, 32)
        bias, hb = rnd(33, (N,), 0.3, BF16)
        gate, hg = rnd(34, (N,), 0.5)
        y, err, _, _ = forward_bounds(host(o, kw), hb, BF16)
        silu = blocks.act("silu", y)
        lin = 1.13 * err + 2.0 ** -20 * (A(y) + err)   # (the activation's slope, its exponential and reciprocal)
        within(t2i.adapter_linear(**o, bias=bias, **kw, epilogue="silu"), silu, U[BF16] * (A(silu) + lin) + lin, "silu")
        resid, hr = rnd(35, (M, N), 2.0)
        buf = torch.full((M + 1, N + 3), 7.0, device=DEV)
        buf[:-1, :N] = resid
        t2i.adapter_linear(**o, bias=bias, **kw, epilogue="resid_gated", resid=buf[:-1, :N], gate=gate)
        ref = hr + hg * y
        within(buf[:-1, :N], ref, A(hg) * err + 3 * E * (A(hg * y) + A(ref)), "resid_gated")
        assert (buf[:-1, N:] == 7).all() and (buf[-1] == 7).all()


def test_the_largest_tiles_are_reached():
    v = [C.c_int() for _ in range(4)]
    tiles = set()
    for op in (4, 5):
        for M, N, K, *_ in SHAPES:
            assert t2i.load().t2i_test_block_tile(op, 1, M, N, K, *map(C.byref, v))
            tiles.add((op, v[0].value, v[1].value))
    say(sorted(tiles))
    assert {(4, 256, 256), (4, 192, 256), (4, 256, 192), (5, 256, 256), (5, 192, 256)} <= tiles


@pytest.mark.parametrize("M,N,K", [(3, 33, 17), (70, 131, 65), (130, 67, 259), (333, 1155, 1153), (17, 1, 3), (66, 3, 1),
                                   (1030, 257, 129)])
@pytest.mark.parametrize("at", [0, 1, 3])
def test_adapters_f32_any_width_and_address(M, N, K, at):
    """Rows off 16 bytes and inside larger buffers, with the gradients."""
    o, kw = operands(M, N, K, 4, 6, "runs", F32, 3)
    h = host(o, kw)
    y, err, _, _ = forward_bounds(h, None, F32)

    def shifted(t):
        buf = torch.full((t.numel() + at,), 7.0, device=DEV)
        buf[at:] = t.reshape(-1)
        return buf[at:].view(t.shape)
    for extra in (0, 3):
        s = {k: shifted(v) for k, v in o.items()}
        if extra:
            s.update({k: padded(o[k], extra)[0] for k in "xw"})
        out, t = t2i.adapter_linear(**s, **kw, save_t=True)
        within(out, y, E * A(y) + err)
        dy, hdy = rnd(8, (M, N), 1.0, F32)
        got = t2i.adapter_linear_backward(padded(dy, extra)[0] if extra else shifted(dy), **s, t=t, **kw)
        ref, bounds = backward_bounds(h, hdy, F32)
        for v, name in zip(got, ("dx", "da", "db")):
            within(v, ref[name], E * A(ref[name]) + bounds[name], name)


@pytest.mark.parametrize("M,N,K", [(1, 72, 304), (5, 128, 128), (70, 1152, 1152), (300, 264, 704), (2050, 2304, 256)])
def test_adapter_epilogues(M, N, K):
    for dtype in (BF16, F32):
        o, kw = operands(M, N, K, 5, 16, "runs", dtype, 4)
        bias, hb = rnd(10, (N,), 0.3, dtype)
        y, err, _, _ = forward_bounds(host(o, kw), hb, dtype)
        for epi in ("gelu", "silu"):
            ref = blocks.act(epi, y)
            # the activations' slopes are at most 1.13; the hardware exponential and reciprocal
            lin = 1.13 * err + 2.0 ** -20 * (A(y) + err)
            within(t2i.adapter_linear(**o, bias=bias, **kw, epilogue=epi), ref, U[dtype] * (A(ref) + lin) + lin, epi)
        gate, rg = rnd(11, (N,), 0.5)
        x0, rx = rnd(12, (M, N), 2.0)
        for epi, g in (("resid", np.ones(N)), ("resid_gated", rg)):
            for copy in (False, True):
                r, buf = padded(x0, 3)
                cp, cbuf = padded(x0.to(BF16), 3)
                before = r._version
                out = t2i.adapter_linear(**o, bias=bias, **kw, epilogue=epi, resid=r, resid_copy=cp if copy else None,
                                         gate=gate if epi == "resid_gated" else None)
                assert out is r and r._version == before + 1
                ref = rx + g * y
                within(r, ref, A(g) * err + 3 * E * (A(g * y) + A(ref)), epi)
                assert (buf[:-1, N:] == 7).all() and (buf[-1] == 7).all()
                if copy:
                    assert torch.equal(cp, r.to(BF16)) and (cbuf[:-1, N:] == 7).all()


@pytest.mark.parametrize("M,N,K,dtype", [(9, 64, 128, BF16), (40, 128, 72, BF16), (300, 264, 200, BF16),
                                         (4000, 4096, 640, BF16), (9, 64, 128, F32), (300, 264, 200, F32)])
def test_one_tenants_nan_stays_with_it(M, N, K, dtype):
    """A NaN or an infinity in an adapter, in its scale or in one row of x reaches the rows that
    take it and no other; the gradients of other adapters neither."""
    for order in ("runs", "scattered"):
        o, kw = operands(M, N, K, 4, 16, order, dtype, 6)
        ix = kw["index"].clone()
        ix[M // 2] = 0     # (adapters 0 and 1 have rows, and row M / 2 is spoiled by itself)
        ix[M // 2 - 1] = 1
        ix[ix == 3] = 2
        kw["index"] = ix
        dy = rnd(8, (M, N), 1.0, dtype)[0]
        y0, t0 = t2i.adapter_linear(**o, **kw, save_t=True)
        g0 = t2i.adapter_linear_backward(dy, **o, t=t0, **kw)
        for where in ("a", "b", "scale", "unused"):
            s, k2 = {k: v.clone() for k, v in o.items()}, dict(kw, scale=kw["scale"].clone())
            if where == "scale":
                k2["scale"][1] = float("nan")
            elif where == "unused":
                s["a"][3], s["b"][3] = float("nan"), float("inf")
            else:
                s[where][1].fill_(float("inf"))
                s[where][1, 0, 0] = float("nan")
            y, t = t2i.adapter_linear(**s, **k2, save_t=True)
            others = ix != 1 if where != "unused" else ix > -9
            assert torch.equal(y[others], y0[others]) and torch.equal(t[others], t0[others])
            assert where == "unused" or not y[~others].isfinite().all(1).any()
            dx, da, db = t2i.adapter_linear_backward(dy, **s, t=t, **k2)
            assert torch.equal(dx[others], g0[0][others])
            keep = [0, 2] if where != "unused" else [0, 1, 2]
            assert torch.equal(da[keep], g0[1][keep]) and torch.equal(db[keep], g0[2][keep])
            assert not da[3].any() and not db[3].any()
        x = o["x"].clone()
        x[M // 2] = float("nan")
        others = torch.arange(M, device=DEV) != M // 2
        y, t = t2i.adapter_linear(**{**o, "x": x}, **kw, save_t=True)
        assert torch.equal(y[others], y0[others]) and y[M // 2].isnan().all()
        dx, da, db = t2i.adapter_linear_backward(dy, **{**o, "x": x}, t=t, **kw)
        assert torch.equal(dx, g0[0]) and torch.equal(da[1:], g0[1][1:]) and torch.equal(db[1:], g0[2][1:])
        assert da[0].isnan().all() and db[0].isnan().all()


@DTYPES
def test_rows_without_an_adapter_are_the_layers(dtype):
    """Bit for bit those of a call in which no row has one; NaN in the padding of t is overwritten."""
    M, N, K = 300, 264, 200
    o, kw = operands(M, N, K, 3, 9, "scattered", dtype, 8)
    kw["index"][::3] = -1
    y = t2i.adapter_linear(**o, **kw)
    none = t2i.adapter_linear(**o, index=torch.full_like(kw["index"], 99), scale=kw["scale"])
    without = (kw["index"] < 0) | (kw["index"] >= 3)
    assert torch.equal(y[without], none[without])
    r = to_host(none) - to_host(o["x"]) @ to_host(o["w"]).T
    assert A(r).max() < 0.05
    lib, st = t2i.load(), C.c_void_p(torch.cuda.current_stream().cuda_stream)
    for rows in (M, 40):
        t = torch.full((rows + 1, 72), float("nan"), device=DEV)
        out = torch.full((rows + 1, N + 5), 7.0, dtype=dtype, device=DEV)
        _lib.check(lib.t2i_op_adapter_linear(
            int(dtype == BF16), 0, rows, N, K, o["x"].data_ptr(), K, o["w"].data_ptr(), K, None, 3, 9, o["a"].data_ptr(),
            o["b"].data_ptr(), kw["scale"].data_ptr(), kw["index"].data_ptr(), t.data_ptr(), 72, out.data_ptr(), N + 5, None,
            0, None, None, st))
        assert torch.equal(out[:rows, :N], t2i.adapter_linear(o["x"][:rows], o["w"], o["a"], o["b"],
                                                              index=kw["index"][:rows], scale=kw["scale"]))
        assert (out[:rows, N:] == 7).all() and (out[rows] == 7).all()
        assert not t[:rows, 9:32].any() and t[:rows, 32:].isnan().all() and t[rows].isnan().all()


# ------------------------------------------------------------------ gradients

def backward_bounds(h, dy, dtype):
    ref = blocks.adapter_linear_grads(dy, **h)
    mag = {**h, **{k: A(h[k]) for k in "xwab"}}
    big = blocks.adapter_linear_grads(A(dy), **mag)
    _, _, t, t_err = forward_bounds(h, None, dtype)
    M, N, K, rank = dy.shape[0], dy.shape[1], h["x"].shape[1], h["a"].shape[1]
    short = 2.0 ** -16 if dtype == BF16 else 0
    u_err, t_err = (N + 2) * E * big["u"] + short * A(ref["u"]), t_err + short * A(t)
    err = dict(dx=(N + 2) * E * (A(dy) @ A(h["w"])) + 4 * E * A(ref["dx"]), da=np.zeros_like(ref["da"]),
               db=np.zeros_like(ref["db"]))
    for i, rows in enumerate(blocks.adapter_rows(h["index"], h["a"].shape[0], M)):
        u = A(ref["u"][rows])
        err["dx"][rows] += (u_err[rows] + (2 * rank + 2) * E * u) @ A(h["a"][i])
        err["da"][i] = (u_err[rows] + (2 * len(rows) + 2) * E * u).T @ A(h["x"][rows])
        err["db"][i] = A(dy[rows]).T @ (t_err[rows] + (2 * len(rows) + 2) * E * A(t[rows]))
    return ref, err


@ORDERS
@CASES
def test_adapter_linear_backward(M, N, K, n, rank, order, dtype):
    n = 1 if order is None else n
    say("adapter bwd", M, N, K, n, rank, order, NAME[dtype])
    o, kw = operands(M, N, K, n, rank, order, dtype, 11)
    dy, hdy = rnd(12, (M, N), 1.0, dtype)
    _, t = t2i.adapter_linear(**o, **kw, save_t=True)
    got = t2i.adapter_linear_backward(dy, **o, t=t, **kw)
    ref, err = backward_bounds(host(o, kw), hdy, dtype)
    for v, name in zip(got, ("dx", "da", "db")):
        assert v.dtype == dtype
        within(v, ref[name], U[dtype] * (A(ref[name]) + err[name]) + err[name], name)
    # each by itself: the same bits
    dx, da, db = t2i.adapter_linear_backward(dy, **o, t=t, **kw, need_dab=False)
    assert torch.equal(dx, got[0]) and da is None and db is None
    dx, da, db = t2i.adapter_linear_backward(dy, **o, t=t, **kw, need_dx=False)
    assert dx is None and torch.equal(da, got[1]) and torch.equal(db, got[2])


@DTYPES
def test_adapters_without_scale_and_without_an_index(dtype):
    """Several adapters and no index: adapter 0 has all rows, the others zeros."""
    o, _ = operands(150, 72, 136, 3, 8, None, dtype, 15)
    dy = rnd(16, (150, 72), 1.0, dtype)[0]
    y, t = t2i.adapter_linear(**o, save_t=True)
    got = t2i.adapter_linear_backward(dy, **o, t=t)
    one = {**o, "a": o["a"][:1].contiguous(), "b": o["b"][:1].contiguous()}
    y1, t1 = t2i.adapter_linear(**one, save_t=True, index=torch.zeros(150, dtype=torch.int32, device=DEV),
                                scale=torch.ones(1, device=DEV))
    ref = t2i.adapter_linear_backward(dy, **one, t=t1, index=torch.zeros(150, dtype=torch.int32, device=DEV))
    assert torch.equal(y, y1) and torch.equal(t, t1) and torch.equal(got[0], ref[0])
    assert torch.equal(got[1][:1], ref[1]) and torch.equal(got[2][:1], ref[2])
    assert not got[1][1:].any() and not got[2][1:].any()
    for g in (t2i.adapter_linear_backward(dy, **o, t=t, index=torch.full((150,), -1, dtype=torch.int32, device=DEV))[1:]):
        assert not g.any()


def test_adapter_gradients_against_differences():
    M, N, K, n, rank = 40, 24, 16, 3, 4
    o, kw = operands(M, N, K, n, rank, "scattered", F32, 17)
    dy = rnd(18, (M, N), 1.0, F32)[0]

    def loss(q):
        return float((to_host(t2i.adapter_linear(**q, **kw)) * to_host(dy)).sum())
    _, t = t2i.adapter_linear(**o, **kw, save_t=True)
    got = dict(zip("xab", t2i.adapter_linear_backward(dy, **o, t=t, **kw)))
    r = np.random.default_rng(19)
    for name in "xab":
        d = dev(r.standard_normal(o[name].shape).astype(np.float32))
        hi, lo = ({**o, name: o[name] + s * d} for s in (2.0 ** -8, -2.0 ** -8))
        num = (loss(hi) - loss(lo)) * 2.0 ** 7
        # y is of first degree in each; 960 values of size about 2 with fp32 errors of (K + rank) E
        assert abs(num - float((to_host(got[name]) * to_host(d)).sum())) < 2.0 ** 7 * 2 * 960 * 2 * 24 * E * 4, name


# ------------------------------------------------------------------ together

def test_adapters_on_another_stream_and_in_graphs():
    """Two graphs of the same calls with workspaces of their own, replayed in turn with eager work between."""
    o, kw = operands(700, 264, 520, 6, 16, "runs", BF16, 21)
    dy = rnd(22, (700, 264), 1.0, BF16)[0]

    def work():
        y, t = t2i.adapter_linear(**o, **kw, save_t=True)
        return (y, t, *t2i.adapter_linear_backward(dy, **o, t=t, **kw))
    ref = [v.clone() for v in work()]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    y = t2i.adapter_linear(**o, **kw, stream=side)
    side.synchronize()
    assert torch.equal(y, ref[0])
    with torch.cuda.stream(side):
        work()
    torch.cuda.synchronize()
    graphs = []
    for _ in range(2):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            graphs.append((graph, work()))
        graphs[-1] = (graph, graphs[-1][1])
    for i in range(4):
        for graph, out in graphs:
            for v in out:
                v.zero_()
            graph.replay()
        torch.cuda.synchronize()
        for _, out in graphs:
            for v, r in zip(out, ref):
                assert torch.equal(v, r)
        work()
        if i == 1:      # other rows' adapters in the same place
            kw["index"].copy_(kw["index"].flip(0))
            ref = [v.clone() for v in work()]


@pytest.mark.parametrize("bad", ["a", "b", "b_strided", "index_type", "index_size", "scale", "dtype", "odd", "epilogue",
                                 "resid", "gate", "t", "host", "rank"])
def test_python_adapter_calls_refuse(bad):
    o, kw = operands(8, 16, 24, 2, 4, "scattered", BF16)
    dy = rnd(3, (8, 16), 1.0, BF16)[0]
    t = torch.zeros((8, 32), device=DEV)
    both = True
    if bad == "a":
        o["a"] = o["a"][:, :, :16]
    elif bad == "b":
        o["b"] = o["b"][:1]
    elif bad == "b_strided":
        o["b"] = o["b"].transpose(1, 2).contiguous().transpose(1, 2)
    elif bad == "index_type":
        kw["index"] = kw["index"].long()
    elif bad == "index_size":
        kw["index"] = kw["index"][:7]
    elif bad == "scale":
        kw["scale"] = kw["scale"].to(BF16)
    elif bad == "dtype":
        o["w"] = o["w"].float()
    elif bad == "odd":
        o["x"], o["w"], o["a"] = (v[..., :20].contiguous() for v in (o["x"], o["w"], o["a"]))
    elif bad == "host":
        o["a"] = o["a"].cpu()
    elif bad == "rank":
        o["a"], o["b"] = torch.zeros((2, 129, 24), dtype=BF16, device=DEV), torch.zeros((2, 16, 129), dtype=BF16, device=DEV)
        t = torch.zeros((8, 160), device=DEV)
    else:
        both = False
    if both:
        with pytest.raises(t2i.T2IError):
            t2i.adapter_linear(**o, **kw)
        with pytest.raises(t2i.T2IError):
            t2i.adapter_linear_backward(dy, **o, t=t, **kw)
    elif bad == "t":
        for wrong in (t[:, :4], t.to(BF16), t[:7]):
            with pytest.raises(t2i.T2IError):
                t2i.adapter_linear_backward(dy, **o, t=wrong, **kw)
    else:
        more = dict(epilogue=dict(epilogue="tanh"), resid=dict(epilogue="resid"), gate=dict(epilogue="resid_gated",
                    resid=torch.zeros((8, 16), device=DEV)))[bad]
        with pytest.raises(t2i.T2IError):
            t2i.adapter_linear(**o, **kw, **more)
