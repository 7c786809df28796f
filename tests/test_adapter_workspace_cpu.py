"""The workspace of the adapters' gradients: what the rows need, not the registered adapters
(nothing here reaches a GPU)."""
import pytest

import paper_2607_26566_amd as t2i
from test_block_ops_cpu import BF16, F32

E = {BF16: 2, F32: 4}


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("M,N,K,rank,n", [(1, 4096, 4096, 4, 32767), (1, 8192, 8192, 1, 512), (700, 1024, 1024, 8, 30000),
                                          (900, 64, 64, 8, 30000), (8192, 4096, 4096, 4, 32767), (4096, 4096, 4096, 16, 4)])
def test_workspace_does_not_grow_with_adapters_that_have_no_rows(dtype, M, N, K, rank, n):
    size = t2i.load().t2i_op_adapter_linear_backward_ws_bytes
    turned = n * (K * ((rank + 7) // 8 * 8) + N * rank) * E[dtype]
    # u and the rows' order; sums of slices of 128 rows and more, two to a slice; dx in 16 slices at most
    rows = M * (128 * 4 + 4) + 16 * M * (K + 4) * 4
    sums = (2 * (M // 128 + 1) * ((rank + 3) // 4 * 4) * (N + K + 16) * 4) if M > 768 else 0
    assert size(dtype, M, N, K, n, rank) <= turned + n * 24 + M + rows + sums + 4096
    # of few rows B is not turned
    if M == 1:
        assert size(dtype, M, N, K, n, rank) <= n * K * ((rank + 7) // 8 * 8) * E[dtype] + n * 24 + rows + 4096
