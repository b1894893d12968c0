"""Registers of the recurrence's, the convolution's and the norms' kernels: what spills costs them twice the time, and the wavefronts that a
SIMD holds are part of how problems are cut."""
import pytest

from test_kernel_resources import _code_objects, _metadata, hip_build, waves_per_simd


@pytest.fixture(scope="module")
def kernels():
    import os

    if not os.path.exists(hip_build.LIB_PATH):
        pytest.skip("the library is not built")
    return {k[".name"]: k for elf in _code_objects(hip_build.LIB_PATH) for k in _metadata(elf)}


@pytest.mark.parametrize("name,waves", [("gated_scan_tokens", 2), ("gated_scan_wide", 3), ("gated_scan_short", 4), ("gated_scan_one_token", 4), ("token_conv_runs", 2),
                                        ("token_conv_backward_runs", 2), ("join_chunks", 4)])
def test_nothing_spills(kernels, name, waves):
    found = {n: k for n, k in kernels.items() if name in n}
    assert found
    for n, k in found.items():
        assert k[".private_segment_fixed_size"] == 0 and waves_per_simd(k) >= waves, n


def test_backward_recurrence(kernels):
    """Two channels to a lane and 16 states, whole: two wavefronts to a SIMD, nothing in scratch."""
    found = {n: k for n, k in kernels.items() if "gated_scan_backward_tokens" in n and "Li4ELi2ELb0ELb0E" in n}
    assert len(found) == 3
    for n, k in found.items():
        assert waves_per_simd(k) == 2, n
        if "If" not in n:  # (twice the registers for what is in flight in fp32)
            assert k[".private_segment_fixed_size"] == 0, n


def test_norms_of_a_row_to_a_wavefront(kernels):
    found = {n: k for n, k in kernels.items() if "residual_norm" in n and "Li1ELb1E" in n}
    assert len(found) == 2 * 5 * 4  # directions, types, loads
    for n, k in found.items():
        assert k[".private_segment_fixed_size"] == 0, n
