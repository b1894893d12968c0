"""The gradients' formulas that the GPU tests compare with, against differentiation and against differences."""
import pytest
import torch

import token_ops_ref as ref


def _leaves(**tensors):
    return {n: None if t is None else t.double().requires_grad_(True) for n, t in tensors.items()}


def _check(loss_of, leaves, got):
    """got[dX] against autograd, and along one direction against (loss(x + h v) - loss(x - h v)) / 2h."""
    given = [n for n in leaves if leaves[n] is not None]
    for n, g in zip(given, torch.autograd.grad(loss_of(leaves), [leaves[n] for n in given])):
        torch.testing.assert_close(got["d" + n], g, rtol=1e-10, atol=1e-10)
        step = 1e-5 * torch.randn(leaves[n].shape, dtype=torch.float64, generator=torch.Generator().manual_seed(1))
        with torch.no_grad():
            ends = [loss_of(leaves | {n: leaves[n] + s * step}) for s in (1, -1)]
        along = (got["d" + n] * step).sum()
        # the third derivative's term, (1e-5)^2 of a value of order one, and 2^-52 of the losses that are subtracted
        assert abs((ends[0] - ends[1]) / 2 - along) <= 1e-7 * (got["d" + n].abs() * step.abs()).sum() + 1e-15 * ends[0].abs()


@pytest.mark.parametrize("skip,gate,bias,first", [(1, 1, 1, 1), (0, 0, 0, 0), (1, 0, 1, 0), (0, 1, 0, 1)])
def test_scan(skip, gate, bias, first):
    g = torch.Generator().manual_seed(3)
    n = lambda *s: torch.randn(*s, generator=g)  # noqa: E731
    B, L, K, N = 2, 7, 3, 5
    v = _leaves(u=n(B, L, K), dt=n(B, L, K) - 1, a=-torch.rand(K, N, generator=g) * 3, b=n(B, L, N), c=n(B, L, N), d=n(K) if skip else None,
                z=n(B, L, K) if gate else None, dt_bias=n(K) if bias else None)
    state, dy = (n(B, K, N).double() if first else None), n(B, L, K).double()
    got = ref.scan_backward(dy, **{k: None if t is None else t.detach() for k, t in v.items()}, state=state)
    _check(lambda leaves: (ref.scan(**leaves, state=state)[0] * dy).sum(), v, got)


@pytest.mark.parametrize("W", [2, 3, 4])
@pytest.mark.parametrize("silu,bias,first", [(True, 1, 1), (False, 0, 0)])
def test_conv(W, silu, bias, first):
    g = torch.Generator().manual_seed(4)
    n = lambda *s: torch.randn(*s, generator=g)  # noqa: E731
    v = _leaves(x=n(2, 6, 3), w=n(3, W), bias=n(3) if bias else None)
    state, dy = (n(2, W - 1, 3).double() if first else None), n(2, 6, 3).double()
    got = ref.conv_backward(dy, **{k: None if t is None else t.detach() for k, t in v.items()}, state=state, silu=silu)
    _check(lambda leaves: (ref.conv(**leaves, state=state, silu=silu)[0] * dy).sum(), v, got)


@pytest.mark.parametrize("G", [None, 1, 2, 6])
@pytest.mark.parametrize("post,residual", [(1, 1), (0, 1), (1, 0)])
def test_norm(G, post, residual):
    g = torch.Generator().manual_seed(5)
    n = lambda *s: torch.randn(*s, generator=g)  # noqa: E731
    M, K = 6, 5
    v = _leaves(h=n(M, K), residual=n(M, K) if residual else None, w=n(K), gate=n(G, K) if G else None, w_post=n(K) if post else None)
    dy, dr = n(M, K).double(), n(M, K).double()

    def loss(leaves):
        y, r = ref.residual_norm(**leaves, scale=0.7)
        return (y * dy).sum() + (r * dr).sum()

    plain = {k: None if t is None else t.detach() for k, t in v.items()}
    r = ref.residual_norm(**plain, scale=0.7)[1]
    plain.pop("residual")
    _check(loss, v, ref.residual_norm_backward(dy, dr, r=r, scale=0.7, **plain))
