"""Buffers that a call would read and write at once, where workgroups share what they read: refused before any launch, on the C boundary's
addresses, which are never read here."""
import pytest
import torch

from test_token_ops_checks import CALLS, P, call, lib  # noqa: F401

pytestmark = pytest.mark.skipif(torch.cuda.is_available(), reason="runs without a GPU")

OVERLAP, HIP = -7, -5
B, L, K, N, W = 2, 5, 48, 16, 4  # of CALLS


def apart(name, **changed):
    """The call with every buffer at an address of its own, far from the others"""
    at = {k: P + (i << 40) for i, (k, v) in enumerate(CALLS[name].items()) if v == P}
    return at | changed


# an output, an input, their row widths (elements of 2 bytes)
PAIRS = [("token_conv", "y", "x", "ldy", "ldx"), ("token_conv_backward", "dx", "x", "lddx", "ldx"), ("token_conv_backward", "dx", "dy", "lddx", "lddy")]


@pytest.mark.parametrize("name,out,into,ld_out,ld_in", PAIRS)
def test_matrices(lib, name, out, into, ld_out, ld_in):  # noqa: F811
    at = apart(name)
    base = at[into]
    rows = B * L
    refused = lambda offset, pitch=K, other=None, **kw: call(lib, name, **(at | {out: base + offset, ld_in: pitch, ld_out: other or pitch} | kw)) == OVERLAP  # noqa: E731
    assert call(lib, name, **at) != OVERLAP  # (no device: the launch fails)
    # the buffer itself, its neighbouring rows, columns of them
    for offset in (0, 2 * K, -2 * K, 2, -2, 2 * K * (rows - 1), -2 * K * (rows - 1)):
        assert refused(offset), offset
    # behind and before it
    for offset in (2 * K * rows, -2 * K * rows):
        assert not refused(offset), offset
    # halves of one wider matrix, either way round; halves that share a column; a row further
    for offset in (2 * K, -2 * K, 2 * K + 2 * 2 * K, -2 * K + 2 * 2 * K * (rows - 1)):
        assert not refused(offset, pitch=2 * K), offset
    for offset in (2 * K - 2, -2 * K + 2, 2 * K + 2, 2 * 2 * K * 3 - 2):
        assert refused(offset, pitch=2 * K), offset
    # pitches that differ: refused where the row ranges meet
    assert refused(0, K, 2 * K) and refused(2 * K * (rows - 1), K, 2 * K) and not refused(2 * K * rows, K, 2 * K)
    # one token to a sequence: each is read by the lanes that write it
    assert not refused(0, L=1) and not refused(2 * K, L=1, B=1)
    assert refused(2 * K, L=1, B=2)  # (another sequence's row)
    # nothing to do, whatever the addresses
    assert not refused(0, B=0)


@pytest.mark.parametrize("name,size", [("gated_scan", 4 * B * K * N), ("token_conv", 2 * B * (W - 1) * K)])
def test_states(lib, name, size):  # noqa: F811
    at = apart(name)
    for offset in (0, 4, -4, size - 4, 4 - size):
        assert call(lib, name, **(at | dict(state_out=at["state"] + offset))) == OVERLAP, offset
    for offset in (size, -size):
        assert call(lib, name, **(at | dict(state_out=at["state"] + offset))) != OVERLAP, offset
    for k in ("state", "state_out"):
        assert call(lib, name, **(at | {k: None})) != OVERLAP


def test_steps_in_place(lib):  # noqa: F811
    for name in ("gated_scan_step", "token_conv_step"):
        at = apart(name)
        assert call(lib, name, **(at | dict(state_out=at["state"]))) != OVERLAP
    at = apart("token_conv_step")
    assert call(lib, "token_conv_step", **(at | dict(y=at["x"]))) != OVERLAP


def test_the_status_has_a_text(lib):  # noqa: F811
    from paper_2412_20386_amd import binding

    assert "overlap" in binding.status_string(OVERLAP)


@pytest.mark.parametrize("name,out,into,ld_out,ld_in", PAIRS)
def test_pitches_beyond_any_matrix(lib, name, out, into, ld_out, ld_in):  # noqa: F811
    """Pitches whose bytes pass 64 bits"""
    at = apart(name)
    for dtype, pitch in ((0, 1 << 62), (2, 1 << 62), (2, 1 << 61), (0, (1 << 63) - 1)):
        kw = dict(dtype=dtype, B=1, L=2)
        assert call(lib, name, **(at | {out: at[into], ld_in: pitch, ld_out: pitch} | kw)) == OVERLAP
        assert call(lib, name, **(at | {out: at[into], ld_in: pitch, ld_out: K} | kw)) == OVERLAP
        assert call(lib, name, **(at | {ld_in: pitch, ld_out: pitch} | kw)) == HIP
