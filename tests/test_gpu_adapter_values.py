"""What the adapters' products make of t's bits and of infinities, on the GPU.

E = 2^-24.  A sum of n products in fp32 is off by at most n E times the sum of the products'
sizes; bf16 operands' t enters the second product with all of its bits, as three bf16 values
(2^-39 of it short), so that a product of `rank` terms has 3 rank of them."""
import numpy as np
import pytest
import torch

import paper_2607_26566_amd as t2i
from oracle import blocks
from gpu_common import DEV, say, to_host
from test_gpu_block_ops import BF16, DTYPES, E, rnd, within

pytestmark = pytest.mark.gpu
A = np.abs

# tiles of 16 to 256 rows, in one adapter and in several
TILES = [(5, 64, 8, 4), (40, 128, 16, 3), (300, 264, 8, 2), (2100, 4608, 8, 4), (4000, 4096, 8, 4), (3600, 3328, 8, 4),
         (4000, 2816, 8, 4)]


def rows_of(order, M, n):
    if order == "runs":
        return torch.arange(M, device=DEV, dtype=torch.int32) * n // M
    return torch.arange(M, device=DEV, dtype=torch.int32) % n


@pytest.mark.parametrize("order", ["runs", "mixed"])
@pytest.mark.parametrize("M,N,K,rank", TILES)
def test_second_products_take_all_bits_of_t(M, N, K, rank, order):
    """Without a layer (W = 0) and added to an fp32 residual of zeros, y is t B^T before any
    rounding to bf16: off by what K + 2 products make of t and 3 rank + 2 of y."""
    say("bits of t", M, N, K, rank, order)
    x, _ = rnd(1, (M, K), 1.0, BF16)
    a, _ = rnd(2, (3, rank, K), 1.0, BF16)
    b, _ = rnd(3, (3, N, rank), 1.0, BF16)
    w = torch.zeros((N, K), dtype=BF16, device=DEV)
    index, scale = rows_of(order, M, 3), torch.tensor([1.1, 0.7, 1.9], device=DEV)
    y = torch.zeros((M, N), device=DEV)
    t2i.adapter_linear(x, w, a, b, index=index, scale=scale, epilogue="resid", resid=y)
    ix = index.cpu().numpy()
    ref, err = np.zeros((M, N)), np.zeros((M, N))
    for i in range(3):
        rows = ix == i
        s = float(scale[i])
        t = s * to_host(x)[rows] @ to_host(a)[i].T
        size = s * A(to_host(x)[rows]) @ A(to_host(a)[i]).T
        ref[rows] = t @ to_host(b)[i].T
        err[rows] = ((K + 2) * E * size + (3 * rank + 2) * E * A(t)) @ A(to_host(b)[i]).T
    within(y, ref, err + E * A(ref), order)


def same_infinities(got, ref, what):
    """ref as IEEE sums have it: the same infinities and NaN, finite elsewhere."""
    got, ref = got.float().cpu(), torch.from_numpy(ref).float()
    for name, f in (("nan", torch.isnan), ("+inf", torch.isposinf), ("-inf", torch.isneginf)):
        assert torch.equal(f(got), f(ref)), (what, name)


@pytest.mark.parametrize("order", ["runs", "mixed"])
@pytest.mark.parametrize("M,N,K,rank", TILES + [(800, 264, 200, 20), (1500, 64, 520, 16)])
@DTYPES
def test_infinities_keep_their_sign(M, N, K, rank, order, dtype):
    """An infinite element of b, a, x or dy makes its sums infinite with the sign of its factor,
    as sums in float64 have it, and NaN only where they have it (0 times it, or both signs)."""
    say("infinities", M, N, K, rank, order, dtype)
    if dtype != BF16 and M > 2100:
        M = 1100
    x, _ = rnd(11, (M, K), 1.0, dtype)
    w, _ = rnd(12, (N, K), K ** -0.5, dtype)
    a, _ = rnd(13, (3, rank, K), 1.0, dtype)
    b, _ = rnd(14, (3, N, rank), 1.0, dtype)
    dy, _ = rnd(15, (M, N), 1.0, dtype)
    x[M // 3] = 0          # (t = 0 there: times an infinity NaN)
    inf = float("inf")
    for where in ("b", "a", "x", "dy", "t"):
        s = dict(x=x.clone(), w=w, a=a.clone(), b=b.clone())
        d = dy.clone()
        if where == "b":
            s["b"][1, N // 2, rank - 1], s["b"][2, 0, 0], s["b"][0, N - 1, 0] = inf, -inf, -inf
        elif where == "a":
            s["a"][1, rank - 1, K // 2], s["a"][2, 0, 0] = inf, -inf
        elif where == "x":
            s["x"][M - 1, K // 2], s["x"][1, 0] = inf, -inf
        elif where == "dy":
            d[M - 1, N // 2], d[1, 0] = inf, -inf
        index = rows_of(order, M, 3)
        kw = dict(index=index, scale=torch.tensor([1.0, 0.5, 1.5], device=DEV))
        h = {k: to_host(v) for k, v in s.items()}
        h.update(index=index.cpu().numpy(), scale=to_host(kw["scale"]))
        y, t = t2i.adapter_linear(**s, **kw, save_t=True)
        with np.errstate(invalid="ignore"):
            ry, rt = blocks.adapter_linear(**h)
        same_infinities(y, ry, (where, "y"))
        same_infinities(t[:, :rank], rt, (where, "t"))
        if where == "t":   # t itself, as no forward pass of these operands leaves it
            t[M - 1, 0], t[1, rank - 1] = inf, -inf
        dx, da, db = t2i.adapter_linear_backward(d, **s, t=t, **kw)
        ht = to_host(t)[:, :rank]
        with np.errstate(invalid="ignore"):
            ref = blocks.adapter_linear_grads(to_host(d), **h)
            rdb = np.zeros(db.shape)
            for i, rows in enumerate(blocks.adapter_rows(h["index"], 3, M)):
                rdb[i] = to_host(d)[rows].T @ ht[rows]
        same_infinities(dx, ref["dx"], (where, "dx"))
        same_infinities(da, ref["da"], (where, "da"))
        same_infinities(db, rdb, (where, "db"))
