"""Widths whose parameters have more than 2^27 gradients: the sums over workgroups go over their columns in several rounds."""
import pytest
import torch

import paper_2412_20386_amd as ptq
import token_ops_ref as ref
from scan_bounds import bounds, within

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
U = 2.0 ** -24


def _drawing(seed):
    g = torch.Generator(device=DEV).manual_seed(seed)
    return lambda *s, scale=1.0, dtype=torch.float32: (torch.randn(*s, generator=g, device=DEV) * scale).to(dtype)


def test_conv():
    K, W, L = (1 << 27) // 5 + 1001, 4, 2
    n = _drawing(1)
    x, dy, w, bias = n(L, K, dtype=torch.float16), n(L, K, dtype=torch.float16), n(K, W), n(K)
    print("conv", K, flush=True)
    dx, dw, dbias = ptq.token_conv_backward(dy, x, w, bias, 1, L, silu=False)
    with torch.device(DEV):
        want = ref.conv_backward(dy.double()[None], x.double()[None], w.double(), bias.double(), None, False)
        size = ref.conv_backward(dy.double()[None], x.double()[None], w.double(), bias.double(), None, False, magnitude=True)
    assert within(dx[None], want["dx"], (W + 1) * U * size["dx"], torch.float16) <= 1
    # a product and a sum for each token, and the sums over lanes that have none (exact)
    assert within(dw, want["dw"], 2 * L * U * size["dw"], torch.float32) <= 1
    assert within(dbias, want["dbias"], L * U * size["dbias"], torch.float32) <= 1
    # no sequences: zeros in every column
    e = torch.empty((0, K), dtype=torch.float16, device=DEV)
    assert all(bool((t == 0).all()) for t in ptq.token_conv_backward(e, e, w, bias, 0, L)[1:])


def test_scan():
    N, L = 64, 2
    K = (1 << 27) // (N + 2) + 101
    n = _drawing(2)
    v = dict(u=n(L, K), dt=n(L, K), a=-n(K, N).abs() - 0.1, b=n(L, N), c=n(L, N), d=n(K), z=n(L, K), dt_bias=n(K) - 2)
    dy, marks = n(L, K), torch.empty((1, 1, K, N), device=DEV)
    print("scan", K, flush=True)
    y = ptq.gated_scan(*v.values(), 1, L, marks=marks)
    grads = ptq.gated_scan_backward(dy, *v.values(), marks, 1, L)
    exact = {k: t.double()[None] if k in ("u", "dt", "b", "c", "z") else t.double() for k, t in v.items()}
    want = bounds(dy.double()[None], **exact)
    got = dict(zip(("du", "ddt", "da", "db", "dc", "dd", "dz", "ddt_bias"), grads), y=y)
    for k, t in got.items():
        t = t.double()
        assert within(t[None] if k in ("y", "du", "ddt", "db", "dc", "dz") else t, *want[k], torch.float32) <= 1, k
