"""The norm's results at the ends of fp32's range and of long sums, on the GPU against float64
definitions (``oracle/blocks.py``).  E = 2^-24, half a step of fp32 relative to the value; values
below 2^-126 lie 2^-149 apart."""
import numpy as np
import pytest
import torch

import paper_2607_26566_amd as t2i
from oracle import blocks
from gpu_common import DEV, say, to_host
from test_gpu_block_ops import BF16, E, F32, rnd, within
from test_gpu_norm_ops import TYPED

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("K", [3, 500, 1000, 1300, 2000, 3000, 6000, 10000, 33000])
@TYPED
def test_codes_of_products_below_the_normal_range(dtype, rtype, K):
    """h w around fp32's smallest values, where a product loses bits that its quotient by the row's
    largest does not: every code within -127 .. 127 and right, T and the scale as T's own bits give
    them; in rows between usual ones and a row of zeros."""
    say("small products", dtype, rtype, K)
    h, _ = rnd(K, (8, K), 1.0, dtype)
    w, _ = rnd(K + 1, (K,), 1.0, dtype)
    size = 2.0 ** torch.tensor([0, -76, -71, 5, -60, -66, -126, -74], dtype=F32, device=DEV)
    h = (h.float() * size[:, None]).to(dtype)
    h[6] = 0
    h[7, 0], w[0] = 1.1875 * 2.0 ** -75, 1.1875
    w = (w.float() * 2.0 ** -74).to(dtype)
    x, resid = (h, None) if rtype is None else (torch.zeros_like(h), h.to(rtype))
    for eps in (1e-6, 0.25):
        for many in (False, True):   # (few rows have more threads each)
            rows = 2100 if many else 8
            xs = x.repeat(rows // 8 + 1, 1)[:rows]
            rs = None if resid is None else resid.repeat(rows // 8 + 1, 1)[:rows]
            q, s, _ = t2i.add_rms_norm_i8(xs, w, rs, eps=eps)
            assert all(torch.equal(q[i], q[i % 8]) and torch.equal(s[i], s[i % 8]) for i in range(8, rows, 177))
            q, s = q[:8].cpu().numpy(), s[:8]
            rq, rsc = blocks.add_rms_norm_i8(to_host(h), to_host(w), eps)
            assert np.array_equal(q[:, :K], rq)
            within(s, rsc, 42 * E * rsc + 2.0 ** -149)
            if K > 1024 and many:
                break


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_scales_of_small_weights_and_of_large_ones(dtype):
    """T below fp32's normal range or near its end, the scale within it."""
    for K in (40, 2100):
        h, _ = rnd(5, (4, K), 1.0, dtype)
        h = (h.float() * 2.0 ** torch.tensor([-10.0, -20, 3, 0], device=DEV)[:, None]).to(dtype)
        for big in (2.0 ** -128, 2.0 ** -131, 2.0 ** 124):
            w = torch.full((K,), big, dtype=dtype, device=DEV)
            w[1::3] = big / 2
            q, s, _ = t2i.add_rms_norm_i8(h[:2] if big > 1 else h, w, eps=0.0)
            rq, rs = blocks.add_rms_norm_i8(to_host(h)[:2] if big > 1 else to_host(h), to_host(w), 0.0)
            assert np.array_equal(q.cpu().numpy()[:, :K], rq)
            within(s, rs, 42 * E * rs + 2.0 ** -149)


# rows of one wave, of a workgroup of one to four pieces per thread, longer ones
@pytest.mark.parametrize("rows,K", [(13, 64), (40000, 64), (20000, 512), (9000, 1000), (6000, 1152), (3000, 4096),
                                    (1400, 8192), (1300, 10000), (900, 16384), (700, 20000)])
def test_weight_gradients_in_fp32_are_sums_in_more(rows, K):
    """With h = +-1 and eps = 0 r is 1 but for its own rounding and that of 1 / K, 2 E and E, the same
    in all rows, and dy n is exact otherwise: dw is off by that and by its last rounding, E, whatever
    it is beside the sizes of what it sums up (fp64: 2^-53 of them for each of the rows)."""
    say("dw", rows, K)
    dy, hdy = rnd(rows, (rows, K), 1.0, F32)
    h = torch.where(rnd(K, (rows, K), 1.0, F32)[0] < 0, -1.0, 1.0)
    w, _ = rnd(K + 1, (K,), 0.3, F32)
    _, _, dw = t2i.add_rms_norm_backward(dy, h, w, eps=0.0)
    terms = hdy * to_host(h)
    ref = terms.sum(0)
    within(dw, ref, 4 * E * np.abs(ref) + 2.0 ** -53 * rows * np.abs(terms).sum(0))
