"""Registers of the kernels of the residual norm, the adapters and AdamW, read from the
metadata of the built library (no GPU needed)."""
import re

from test_kernel_resources_cpu import find, kernels  # noqa: F401


def test_norm_and_optimizer_kernels_do_not_spill(kernels):  # noqa: F811
    for name in ("add_rms_norm_kernel", "add_rms_norm_bwd_kernel", "add_rms_norm_bwd_long_kernel",
                 "add_rms_norm_dw_long_kernel", "norm_weight_grad_kernel", "adamw_kernel"):
        for k, v in find(kernels, name).items():
            assert v["vgpr_spill_count"] == 0 and v["private_segment_fixed_size"] == 0, (k, v)


def test_adapter_tiles_leave_registers_for_the_waves_that_lds_holds(kernels):  # noqa: F811
    """512 registers of a SIMD, allotted in eights: two workgroups of 128 x 128 with two stages on a
    CU are four waves, three of 64 x 128 six; only the largest tile spills, before and after its
    loop."""
    waves = {(256, 256, 2): 2, (192, 256, 2): 2, (256, 192, 2): 2, (128, 128, 2): 4, (64, 128, 2): 6}
    for name in ("adapter_linear_kernel", "adapter_dx_kernel"):
        for k, v in find(kernels, name).items():
            bm, bn, _, _, st = map(int, re.search(r"TileDimsILi(\d+)ELi(\d+)ELi(\d+)ELi(\d+)ELi(\d+)E", k).groups())
            assert (v["vgpr_count"] + 7) // 8 * 8 * waves.get((bm, bn, st), 1) <= 512, (k, v)
            assert v["vgpr_spill_count"] <= (40 if (bm, bn) == (256, 256) else 0), (k, v)
    for name in ("adapter_down_kernel", "adapter_down_rows_kernel", "adapter_prepare_kernel", "adapter_outer_kernel",
                 "adapter_sum_kernel"):
        for k, v in find(kernels, name).items():
            assert v["vgpr_spill_count"] == 0 and v["private_segment_fixed_size"] == 0, (k, v)
