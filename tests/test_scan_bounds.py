"""The recurrence's error bounds themselves, on the CPU: their values are those of the plain formulas, they hold for the same sums in 32 bits, and a
decay over a chunk that is held in 16 bits falls out of them."""
import pytest
import torch

import token_ops_ref as ref
from scan_bounds import bounds, within


def _inputs(B, L, K, N, state=True):
    g = torch.Generator().manual_seed(L + K)
    n = lambda *s, scale=1.0: (torch.randn(*s, generator=g) * scale).double()  # noqa: E731
    v = dict(u=n(B, L, K), dt=n(B, L, K, scale=0.7), a=-torch.arange(1, N + 1).double() * torch.exp(n(K, N, scale=0.3)) * 0.5, b=n(B, L, N), c=n(B, L, N), d=n(K),
             z=n(B, L, K), dt_bias=n(K) - 2)
    v = {k: t.float().double() for k, t in v.items()}
    return v, n(B, L, K).float().double(), (n(B, K, N).float().double() if state else None)


@pytest.mark.parametrize("state", [False, True])
def test_values(state):
    v, dy, first = _inputs(2, 37, 6, 5, state)
    out = bounds(dy, **v, state=first)
    y, h, _ = ref.scan(**v, state=first)
    want = dict(ref.scan_backward(dy, **v, state=first), y=y, state_out=h[:, -1], marks=h[:, :37:8].transpose(0, 1))
    assert set(out) == set(want)
    for k, t in want.items():
        assert torch.allclose(out[k][0], t, rtol=1e-11, atol=1e-12), k
        assert (out[k][1] > 0).any() and (out[k][1] < 1e-2 * (1 + t.abs().max())).all(), k


def _in_chunks(v, state, chunk, sum_type):
    """States behind every chunk as chunks give them that run from zero and are joined, each chunk's sum of D held in `sum_type`."""
    D = ref.softplus(v["dt"] + v["dt_bias"])
    B, L, K = D.shape
    h, states = state, []
    for t0 in range(0, L, chunk):
        at = slice(t0, t0 + chunk)
        part = {k: (t[:, at] if k in ("u", "dt", "b", "c", "z") else t) for k, t in v.items()}
        end = ref.scan(**part)[1][:, -1]
        total = D[:, at].sum(1).to(sum_type).double()
        h = torch.exp(v["a"] * total[..., None]) * h + end
        states.append(h)
    return torch.stack(states)


def test_a_long_sequence_in_chunks():
    v, dy, first = _inputs(1, 1600, 6, 4)
    v["a"] /= 8  # (what a state carries over a chunk of 32 tokens is to count)
    out = bounds(dy, **v, state=first)
    want, error = torch.cat([out["marks"][0][4::4], out["state_out"][0][None]]), torch.cat([out["marks"][1][4::4], out["state_out"][1][None]])
    assert within(_in_chunks(v, first, 32, torch.float32), want, error, torch.float32) <= 1
    assert within(_in_chunks(v, first, 32, torch.bfloat16), want, error, torch.float32) > 2


def test_the_plain_recurrence_in_32_bits():
    v, dy, first = _inputs(2, 300, 5, 4)
    out = bounds(dy, **v, state=first, chunk=300)
    s = {k: t.float() for k, t in v.items()}
    h, parts = first.float(), []
    D = ref.softplus(s["dt"] + s["dt_bias"])
    for t in range(300):
        h = torch.exp(D[:, t, :, None] * s["a"]) * h + (D * s["u"])[:, t, :, None] * s["b"][:, t, None, :]
        parts.append((h * s["c"][:, t, None, :]).sum(-1) + s["d"] * s["u"][:, t])
    y = torch.stack(parts, 1) * s["z"] * ref.sigmoid(s["z"])
    assert within(y, *out["y"], torch.float32) <= 1
    assert within(h, *out["state_out"], torch.float32) <= 1
