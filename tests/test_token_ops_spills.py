"""What every kernel of the recurrence, the convolution and the norms keeps in scratch: nothing, but for the layouts named here, whose rows or states do not
fit the registers that their wavefronts leave them."""
import os

import pytest

from test_kernel_resources import _code_objects, _metadata, hip_build

KERNELS = ("gated_scan_", "join_chunks", "sum_column_blocks", "sum_partials", "sum_norm_partials", "token_conv_", "residual_norm_")
# part of a kernel's name: bytes a lane that are accepted
SPILLS = {
    "residual_norm_rowsIDF16_DF16_Li8ELi2ELi16E": 72, "residual_norm_rowsIDF16_fLi8ELi2ELi16E": 72, "residual_norm_rowsIDF16bDF16bLi8ELi2ELi16E": 72,
    "residual_norm_rowsIDF16bfLi8ELi2ELi16E": 72, "residual_norm_rowsIffLi8ELi2ELi16E": 72,  # 8193 columns and more: 16 wavefronts of two loads
    **{f"residual_norm_backward_rowsI{t}Li8ELi2ELi{waves}E": n for t in ("DF16_DF16_", "DF16_f", "DF16bDF16b", "DF16bf", "ff")
       for waves, n in ((8, 100), (16, 700))},  # 4097 columns and more
    "gated_scan_backward_tokensIDF16_Li4ELi1ELb0ELb0E": 12, "gated_scan_backward_tokensIDF16bLi4ELi1ELb0ELb0E": 12,  # one channel to a lane, 16 states
    "gated_scan_backward_tokensIfLi4ELi1ELb0ELb0E": 24, "gated_scan_backward_tokensIfLi4ELi1ELb1ELb0E": 24,
    "gated_scan_backward_tokensIfLi4ELi2ELb0ELb0E": 28, "gated_scan_backward_tokensIfLi4ELi2ELb1ELb0E": 28,  # fp32: twice what is in flight
}


@pytest.fixture(scope="module")
def kernels():
    if not os.path.exists(hip_build.LIB_PATH):
        pytest.skip("the library is not built")
    found = {k[".name"]: k[".private_segment_fixed_size"] for elf in _code_objects(hip_build.LIB_PATH) for k in _metadata(elf)}
    return {n: size for n, size in found.items() if any(k in n for k in KERNELS)}


def test_every_kernel(kernels):
    # types x layouts (states and channels to a lane; taps; loads, elements and wavefronts of a row) x the variants with and without bounds, and so on
    for name, count in (("gated_scan_tokensI", 3 * 8 * 4), ("gated_scan_backward_tokensI", 3 * 8 * 4), ("gated_scan_wideI", 6), ("gated_scan_shortI", 6),
                        ("gated_scan_one_tokenI", 3 * 6 * 2), ("token_conv_runsI", 18), ("token_conv_backward_runsI", 18), ("residual_norm_rowsI", 5 * 12),
                        ("residual_norm_backward_rowsI", 5 * 12)):
        assert sum(name in n for n in kernels) == count, name
    for n, size in kernels.items():
        assert size <= max([most for part, most in SPILLS.items() if part in n], default=0), (n, size)


def test_the_list_holds_no_others(kernels):
    for part in SPILLS:
        assert any(part in n and size > 0 for n, size in kernels.items()), part
