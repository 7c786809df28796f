"""The sizes of ``adapter_tiles`` take the kernels they stand for, and no size takes another
(nothing here reaches a GPU)."""
import math
import random

from adapter_tiles import DX, FWD, SIZES, kernel_of


def test_each_size_takes_its_kernel():
    for key, size in SIZES.items():
        assert kernel_of(key[0], key[1], *size) == key, size


def test_no_size_takes_a_kernel_that_is_not_run():
    r = random.Random(3)

    def log(lo, hi):
        return int(round(math.exp(r.uniform(math.log(lo), math.log(hi)))))
    for _ in range(40000):
        dtype = r.choice(["bf16", "f32"])
        M, N, K = log(1, 20000), 8 * log(1, 2500), 8 * log(1, 1500)
        if dtype == "f32":
            N, K = N + r.choice([0, 0, 1, 3]), K + r.choice([0, 0, 1, 3])
        for product in (FWD, DX):
            assert kernel_of(product, dtype, M, N, K) in SIZES, (product, dtype, M, N, K)
