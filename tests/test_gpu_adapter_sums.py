"""The adapters' gradient sums where an adapter's rows begin and end: on the borders of the slices
they are cut into, beside them, in one slice or many, with many adapters that have none.  Bounds as
in test_gpu_adapters."""
import numpy as np
import pytest
import torch

import paper_2607_26566_amd as t2i
from gpu_common import DEV, say
from test_gpu_adapters import check_all, operands
from test_gpu_block_ops import BF16, DTYPES, F32, rnd

pytestmark = pytest.mark.gpu


def by_counts(counts, M, n, seed):
    """adapters with so many rows each one after the other, the rows left over without; then the
    rows shuffled"""
    ix = np.full(M, -1)
    at = 0
    for i, c in counts:
        ix[at:at + c] = i
        at += c
    assert at <= M and max(i for i, _ in counts) < n
    return ix, np.random.default_rng(seed).permutation(ix)


# slices have 128 rows at N = K = 64 (of as many adapters as in the last case 1024)
CASES = [
    (1024, 9, [(0, 128), (2, 128), (3, 256), (5, 1), (7, 127), (8, 384)]),       # on the borders
    (1100, 12, [(1, 127), (2, 1), (4, 129), (5, 126), (6, 2), (9, 383), (11, 200)]),
    (896, 3, [(1, 896)]),                                                       # all rows one adapter's
    (900, 4, [(3, 128)]),                                                       # most without
    (1500, 6, [(0, 1), (5, 1499)]),
    (1500, 6, [(0, 1499), (5, 1)]),
    (1024, 30000, [(7, 200), (8, 56), (9, 128), (20000, 300), (29999, 340)]),    # many more adapters than rows
]


@pytest.mark.parametrize("case", range(len(CASES)))
@DTYPES
def test_sums_of_adapters_on_the_borders_of_slices(case, dtype):
    M, n, counts = CASES[case]
    N = K = 64
    say("borders", M, n, dtype)
    o, kw = operands(M, N, K, n, 3, "one", dtype, 41)
    for ix in by_counts(counts, M, n, case):
        kw["index"] = torch.from_numpy(ix.astype(np.int32)).to(DEV)
        check_all(o, kw, M, N, dtype, 42)


@pytest.mark.parametrize("M,N,K,n,rank", [(900, 64, 64, 900, 5), (1100, 64, 72, 2500, 3), (2100, 2304, 1152, 7, 40),
                                          (1024, 4608, 4096, 3, 20), (1030, 4608, 4096, 1, 20)])
@DTYPES
def test_sums_of_a_row_each_and_of_wide_layers(M, N, K, n, rank, dtype):
    """More adapters than slices, every row another's; slices of 128 to 1024 rows."""
    for order in (("scattered", "runs", None) if n < 10 else ("scattered",)):
        o, kw = operands(M, N, K, 1 if order is None else n, rank, order, dtype, 43)
        check_all(o, kw, M, N, dtype, 44)


def test_one_row_among_all_the_adapters_there_may_be():
    M, N, K, n = 1, 64, 64, 32767
    o, kw = operands(M, N, K, n, 1, "one", BF16, 45)
    kw["index"][0] = 777
    dy = rnd(46, (M, N), 1.0, BF16)[0]
    _, t = t2i.adapter_linear(**o, **kw, save_t=True)
    torch.cuda.synchronize()
    before = torch.cuda.memory_allocated()
    torch.cuda.reset_peak_memory_stats()
    dx, da, db = t2i.adapter_linear_backward(dy, **o, t=t, **kw)
    torch.cuda.synchronize()
    grads = 2 * n * 64 * 2
    assert torch.cuda.max_memory_allocated() - before < grads + n * (64 * 8 * 2 + 24) + (1 << 20)
    rows = torch.arange(n, device=DEV) != 777
    assert not da[rows].any() and not db[rows].any() and da[777].any() and db[777].any()


@pytest.mark.parametrize("M", [1023, 1024, 1025, 2048, 2049])
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_one_slice_and_a_row_more_without_an_index(M, dtype):
    """Adapter 0 has all rows, the others zeros; the same bits as with an index."""
    N, K = 4608, 4096
    o, kw = operands(M, N, K, 3, 8, "one", dtype, 47)
    kw["index"].zero_()
    dy = rnd(48, (M, N), 1.0, dtype)[0]
    _, t = t2i.adapter_linear(**o, **kw, save_t=True)
    ref = t2i.adapter_linear_backward(dy, **o, t=t, **kw)
    kw["index"] = None
    got = t2i.adapter_linear_backward(dy, **o, t=t, **kw)
    assert all(torch.equal(a, b) for a, b in zip(got, ref))
    assert not got[1][1:].any() and not got[2][1:].any() and got[1][0].any()
