"""The limits that the header names, from both sides: on the C boundary, where a call that passes them finds no device to launch on."""
import pytest
import torch

from test_token_ops_checks import CALLS, P, SHAPE, STRIDE, lib  # noqa: F401

pytestmark = pytest.mark.skipif(torch.cuda.is_available(), reason="runs without a GPU")
HIP = -5


def _call(lib, name, **changed):  # noqa: F811
    """With pitches of the rows' widths, unless they are given"""
    sizes = CALLS[name] | changed
    pitches = {k: sizes["N"] if k in ("ldb", "ldc", "lddb", "lddc") else sizes["K"] for k in sizes if k.startswith("ld")}
    at = {k: P + (i << 56) for i, (k, v) in enumerate(CALLS[name].items()) if v == P}  # (none of these sizes reaches the next buffer)
    return getattr(lib, "ptq4vm_" + name)(*(CALLS[name] | at | pitches | changed).values())


# entry point, sizes inside and beyond each limit, the status beyond
LIMITS = [
    ("gated_scan", dict(B=1, K=(1 << 23) - 1), dict(B=1, K=1 << 23), SHAPE),
    ("gated_scan", dict(B=(1 << 25) - 1, K=16), dict(B=1 << 25, K=16), SHAPE),
    ("gated_scan", dict(N=64), dict(N=65), SHAPE),
    ("gated_scan", dict(B=1, L=(1 << 31) - 1), dict(B=1, L=1 << 31), SHAPE),
    ("gated_scan", dict(ldu=(1 << 26) - 1), dict(ldu=1 << 26), STRIDE),
    ("gated_scan_backward", dict(B=1, K=(1 << 23) - 1), dict(B=1, K=1 << 23), SHAPE),
    ("gated_scan_backward", dict(B=(1 << 25) - 1, K=16), dict(B=1 << 25, K=16), SHAPE),
    ("gated_scan_backward", dict(lddz=(1 << 26) - 1), dict(lddz=1 << 26), STRIDE),
    ("gated_scan_step", dict(B=(1 << 24) - 1, K=16), dict(B=1 << 24, K=16), SHAPE),
    ("token_conv", dict(B=1, L=1, K=(1 << 27) - 1), dict(B=1, L=1, K=1 << 27), SHAPE),
    ("token_conv_backward", dict(B=1, L=1, K=(1 << 27) - 1), dict(B=1, L=1, K=1 << 27), SHAPE),
    ("residual_norm", dict(K=16384), dict(K=16385), SHAPE),
    ("residual_norm", dict(M=(1 << 31) - 2), dict(M=1 << 31), SHAPE),
    ("residual_norm_backward", dict(M=(1 << 31) - 2), dict(M=1 << 31), SHAPE),
]


@pytest.mark.parametrize("name,inside,beyond,status", LIMITS, ids=str)
def test_limits(lib, name, inside, beyond, status):  # noqa: F811
    if "L" in CALLS[name]:
        inside, beyond = dict(L=1) | inside, dict(L=1) | beyond
    assert _call(lib, name, **inside) == HIP
    assert _call(lib, name, **beyond) == status
