"""Registers of the compiled kernels whose speed rests on several waves per
SIMD, read from the metadata of the built library (no GPU needed)."""
import os
import re
import struct
import subprocess

import pytest

from paper_2607_26566_amd.build import LIB

READELF = "/opt/rocm/llvm/bin/llvm-readelf"
MAGIC = b"__CLANG_OFFLOAD_BUNDLE__"


@pytest.fixture(scope="module")
def kernels(tmp_path_factory):
    """symbol -> {vgpr_count, vgpr_spill_count} of every gfx950 kernel."""
    d = tmp_path_factory.mktemp("code")
    fat = str(d / "fatbin")
    subprocess.run(["objcopy", "-O", "binary", "--only-section=.hip_fatbin", LIB, fat], check=True)
    data, out = open(fat, "rb").read(), {}
    for at in (m.start() for m in re.finditer(re.escape(MAGIC), data)):
        entry = at + len(MAGIC) + 8
        for _ in range(struct.unpack_from("<Q", data, entry - 8)[0]):
            off, size, n = struct.unpack_from("<QQQ", data, entry)
            if b"gfx950" in data[entry + 24:entry + 24 + n]:
                co = str(d / "object")
                with open(co, "wb") as f:
                    f.write(data[at + off:at + off + size])
                notes = subprocess.run([READELF, "--notes", co], check=True, capture_output=True,
                                       text=True).stdout
                for block in re.split(r"\n  - ", notes):
                    sym = re.search(r"\.symbol:\s+(\S+)\.kd", block)
                    if sym:
                        out[sym[1]] = {k: int(re.search(rf"\.{k}:\s+(\d+)", block)[1])
                                       for k in ("vgpr_count", "vgpr_spill_count",
                                                 "private_segment_fixed_size")}
            entry += 24 + n
    assert os.path.getsize(fat) and out
    return out


def find(kernels, name):
    got = {k: v for k, v in kernels.items() if name in k}
    assert got, name
    return got


# the conditioning table streams every adaLN weight: it needs 5 waves per SIMD
# (512 registers, allotted in eights) in flight, as much as 8 rows x 4 columns allow
def test_conditioning_rows_keep_five_waves_per_simd(kernels):
    for k, v in {**find(kernels, "linear_rows_group_kernel"), **find(kernels, "linear_rows_kernel")}.items():
        assert (v["vgpr_count"] + 7) // 8 * 8 * 5 <= 512, (k, v)
        assert v["vgpr_spill_count"] == 0, (k, v)


def test_cache_signal_does_not_spill(kernels):
    for k, v in find(kernels, "cache_signal_kernel").items():
        assert v["vgpr_spill_count"] == 0 and v["private_segment_fixed_size"] == 0, (k, v)


def test_no_head_norm_kernel_that_no_call_reaches(kernels):
    """Halves need head_dim % 16 == 0: no head of 8 (one lane) or 72 (nine lanes)."""
    forms = {k: re.search(r"kernelI(f|DF16b)Li(\d+)ELb([01])ELi\d+E", k)
             for k in {**find(kernels, "qk_norm_rope_kernel"), **find(kernels, "qk_norm_rope_bwd_kernel")}}
    assert all(forms.values())
    assert {int(m[2]) for m in forms.values() if m[3] == "1"} == {2, 4, 8, 16, 32}
    assert {int(m[2]) for m in forms.values() if m[3] == "0"} == {1, 2, 4, 8, 9, 16, 32}


def test_block_operators_keep_their_registers(kernels):
    """No spills but two registers of the widest dW tile, no scratch memory but that and
    the head norms' three dwords (part of the rotation)."""
    for name in ("linear_i8_kernel", "gated_linear_kernel", "gated_dx_kernel", "gated_dw_kernel", "split_sum_kernel",
                 "quant_rows_kernel", "gate_grad_kernel", "gate_bias_grad_kernel", "qk_norm_rope_kernel",
                 "qk_norm_rope_bwd_kernel", "qk_weight_grad_kernel"):
        for k, v in find(kernels, name).items():
            wide = name == "gated_dw_kernel" and "TileDimsILi256E" in k
            assert v["vgpr_spill_count"] <= (2 if wide else 0), (k, v)
            assert v["private_segment_fixed_size"] <= (12 if wide or "qk_norm_rope" in name else 0), (k, v)
