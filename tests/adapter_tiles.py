"""Sizes that take each of the kernels which the adapters' products choose between, one per
kernel: (product, type, operands in whole 16-byte pieces, tile, workgroups to a CU, how the
contraction is shared) -> (M, N, K).  ``how``: by one workgroup's waves together, by groups
of waves, or in slices added up by a second launch."""
import ctypes as C

import paper_2607_26566_amd as t2i

FWD, DX = 4, 5
SIZES = {
    (FWD, "bf16", True, (16, 16), 1, "groups"): (20, 24, 456),
    (FWD, "bf16", True, (16, 32), 2, "groups"): (20, 24, 200),
    (FWD, "bf16", True, (32, 64), 2, "groups"): (353, 360, 200),
    (FWD, "bf16", True, (32, 128), 1, "one"): (20, 16424, 24),
    (FWD, "bf16", True, (32, 128), 2, "one"): (20, 24, 24),
    (FWD, "bf16", True, (64, 128), 2, "one"): (8210, 136, 24),
    (FWD, "bf16", True, (64, 128), 3, "one"): (8875, 264, 72),
    (FWD, "bf16", True, (128, 128), 1, "one"): (718, 5016, 1768),
    (FWD, "bf16", True, (128, 128), 2, "one"): (322, 16544, 24),
    (FWD, "bf16", True, (192, 256), 1, "one"): (5985, 1928, 712),
    (FWD, "bf16", True, (256, 192), 1, "one"): (5764, 2056, 600),
    (FWD, "bf16", True, (256, 256), 1, "one"): (5855, 2808, 456),
    (FWD, "f32", False, (16, 32), 2, "groups"): (20, 25, 129),
    (FWD, "f32", False, (32, 64), 1, "groups"): (20, 25, 97),
    (FWD, "f32", False, (32, 64), 1, "one"): (20, 24, 25),
    (FWD, "f32", False, (64, 64), 1, "one"): (4099, 65, 25),
    (FWD, "f32", False, (128, 128), 1, "one"): (197, 12411, 25),
    (FWD, "f32", True, (16, 32), 2, "groups"): (20, 24, 136),
    (FWD, "f32", True, (32, 64), 1, "groups"): (20, 24, 104),
    (FWD, "f32", True, (32, 64), 1, "one"): (20, 24, 24),
    (FWD, "f32", True, (64, 64), 1, "one"): (8193, 24, 24),
    (FWD, "f32", True, (128, 128), 1, "one"): (1709, 4552, 552),
    (DX, "bf16", True, (16, 32), 2, "groups"): (20, 200, 24),
    (DX, "bf16", True, (32, 64), 2, "groups"): (529, 200, 328),
    (DX, "bf16", True, (32, 128), 2, "one"): (20, 24, 24),
    (DX, "bf16", True, (32, 128), 2, "slices"): (20, 3144, 24),
    (DX, "bf16", True, (64, 128), 2, "one"): (8200, 24, 136),
    (DX, "bf16", True, (64, 128), 2, "slices"): (582, 3360, 392),
    (DX, "bf16", True, (64, 128), 3, "one"): (7578, 24, 392),
    (DX, "bf16", True, (64, 128), 3, "slices"): (1667, 7048, 24),
    (DX, "bf16", True, (128, 128), 1, "one"): (1546, 528, 2312),
    (DX, "bf16", True, (128, 128), 1, "slices"): (963, 5016, 792),
    (DX, "bf16", True, (128, 128), 2, "one"): (2528, 408, 5952),
    (DX, "bf16", True, (128, 128), 2, "slices"): (1733, 6080, 784),
    (DX, "bf16", True, (192, 256), 1, "one"): (6678, 736, 1672),
    (DX, "bf16", True, (256, 256), 1, "one"): (5793, 464, 2736),
    (DX, "bf16", True, (256, 256), 1, "slices"): (390, 16832, 6184),
    (DX, "f32", False, (16, 32), 2, "groups"): (20, 257, 25),
    (DX, "f32", False, (32, 64), 1, "groups"): (20, 161, 25),
    (DX, "f32", False, (32, 64), 1, "one"): (20, 24, 25),
    (DX, "f32", False, (32, 64), 1, "slices"): (20, 1283, 25),
    (DX, "f32", False, (64, 64), 1, "one"): (4097, 25, 65),
    (DX, "f32", False, (64, 64), 1, "slices"): (194, 1955, 193),
    (DX, "f32", False, (128, 128), 1, "one"): (2181, 25, 1345),
    (DX, "f32", False, (128, 128), 1, "slices"): (251, 2401, 2059),
    (DX, "f32", True, (16, 32), 2, "groups"): (20, 264, 24),
    (DX, "f32", True, (32, 64), 1, "groups"): (20, 168, 24),
    (DX, "f32", True, (32, 64), 1, "one"): (20, 24, 24),
    (DX, "f32", True, (32, 64), 1, "slices"): (20, 1288, 24),
    (DX, "f32", True, (64, 64), 1, "one"): (8193, 24, 24),
    (DX, "f32", True, (64, 64), 1, "slices"): (452, 1936, 72),
    (DX, "f32", True, (128, 128), 1, "one"): (7334, 488, 400),
    (DX, "f32", True, (128, 128), 1, "slices"): (2839, 4848, 104),
}


def kernel_of(product, dtype, M, N, K):
    """The key of a call's kernel, from the library's own choice."""
    v = [C.c_int() for _ in range(4)]
    assert t2i.load().t2i_test_block_tile(product, int(dtype == "bf16"), M, N, K, *map(C.byref, v))
    rows, columns, per_cu, shares = (x.value for x in v)
    tile, how = (rows, columns), "one"
    if shares > 1:   # (fp32 tiles of 32 x 64 have two groups; slices of theirs are more than two here)
        groups = tile in ((16, 16), (16, 32)) or (tile == (32, 64) and (dtype == "bf16" or shares == 2))
        how = "groups" if groups else "slices"
    return product, dtype, dtype == "bf16" or (N % 4 == 0 and K % 4 == 0), tile, per_cu, how
