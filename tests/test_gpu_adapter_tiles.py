"""Every kernel that the adapters' products choose between, with rows in runs and each with
another adapter, against the float64 definitions; bounds as in test_gpu_adapters (slices of a
contraction add up in fp32: no more additions than its length)."""
import pytest

from adapter_tiles import SIZES
from gpu_common import say
from test_gpu_adapters import check_all, operands
from test_gpu_block_ops import BF16, F32

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("key", SIZES, ids=lambda k: "-".join(map(str, k)).replace(" ", ""))
def test_every_tile(key):
    M, N, K = SIZES[key]
    dtype = BF16 if key[1] == "bf16" else F32
    say("tile", *key, M, N, K)
    # (a rank off whole pieces, and one of two steps; the slowest reference only once)
    for rank, order in ((36, "scattered"),) if M * N * K > 2e10 else ((5, "runs"), (36, "scattered")):
        o, kw = operands(M, N, K, 3, rank, order, dtype, 51)
        check_all(o, kw, M, N, dtype, 52)
