"""The gated recurrence and its gradients in 64 bits, each with how far a result in 32 bits may be off: the errors go through the
recurrence with the states, so they are forgotten as the states are, and a long sequence has no wider bounds than a short one.

U is half a step of fp32, one rounding.  With x = dt + dt_bias (a sum: |x| U), e^-|x| (constant, product and instruction: 2 |x| + 2) and
the logarithm of 1 + e^-|x| (6), D is off by (8 + 3 |x|) U of itself; a decay e^{D a} by |D a| times that of D, of a log2(e) and their product
(3), of a sum over the S tokens of a chunk (S, and 16 runs) where it is taken for all of them together, and 2 for the instruction.  A state then takes over
the error of the one before times the decay, and adds those of the decay, of D u b (2) and of its own sum.  `magnitude` values have every
term's absolute value: they bound the states that a chunk reaches from zero too.

Below 2^-126 a rounding is no part of the value: the smallest step is 2^-149, so that each rounding there is off by up to 2^-150 (TINY), and a decay
below 2^-126 (FLUSHED) comes from the instruction as 0.  Both are added as they are, for every product and every sum: 3 a token to a state (the product D u b, the
multiply-add, the join's second product), 2 a term to a sum of products, and a few to what is made of the sums.
"""
import torch

from token_ops_ref import U, sigmoid, softplus

TINY, FLUSHED = 2.0 ** -150, 2.0 ** -126


def bounds(dy, u, dt, a, b, c, d, z, dt_bias, state=None, chunk=160):
    """{result: (value, error)} of the forward and the backward pass; rows [B, L, X] in the order of time, in 64 bits, on the inputs' device.
    `chunk`: at least the tokens that one wavefront runs through."""
    B, L, K = u.shape
    N = a.shape[1]
    new = lambda *s: torch.zeros(*s, dtype=torch.float64, device=u.device)  # noqa: E731
    x = dt + (0 if dt_bias is None else dt_bias)
    D = softplus(x)
    e_D, e_sig = (8 + 3 * x.abs()) * U, (8 + 3 * x.abs()) * U
    gate, e_gate = (torch.ones_like(u), new(B, L, K)) if z is None else (z * sigmoid(z), (2 * z.abs() + 8) * U)
    skip = new(K) if d is None else d
    # of sums over channels: 2 of a lane, 4 over a wavefront, one a column block; over tokens: a chunk's, then the rows of 32 slots
    by_k, by_t = (K / 16 + 16) * U, (chunk + B * L / 24 / 32 + 40) * U
    h, m, e_h = (new(L + 1, B, K, N) for _ in range(3))
    if state is not None:
        h[0], m[0] = state, state.abs()

    def decay(t):
        p = D[:, t, :, None] * a
        return torch.exp(p), p.abs() * (e_D[:, t, :, None] + (3 + chunk + 16) * U) + 3 * U

    y, s, e_s, s_size = (new(B, L, K) for _ in range(4))
    for t in range(L):
        A, e_A = decay(t)
        q = (D * u)[:, t, :, None] * b[:, t, None, :]
        h[t + 1], m[t + 1] = A * h[t] + q, A * m[t] + q.abs()
        e_h[t + 1] = A * e_h[t] + (e_A * A + FLUSHED) * m[t] + (e_D[:, t, :, None] + 2 * U) * q.abs() + U * m[t + 1] + 3 * TINY
        C = c[:, t, None, :]
        s[:, t] = (C * h[t + 1]).sum(-1) + skip * u[:, t]
        size = (C.abs() * m[t + 1]).sum(-1)
        s_size[:, t] = size + (skip * u[:, t]).abs()
        e_s[:, t] = (C.abs() * e_h[t + 1]).sum(-1) + (N + 2) * U * size + U * s_size[:, t] + (2 * N + 4) * TINY
    out = dict(y=(s * gate, e_s * gate.abs() + (e_gate + U) * s_size * gate.abs() + 3 * TINY), state_out=(h[L], e_h[L]), marks=(h[:L:8], e_h[:L:8]))

    G, e_G = dy * gate, e_gate + U
    du, ddt, e_du, e_ddt, size_ddt = (new(B, L, K) for _ in range(5))
    db, dc, e_db, e_dc = (new(B, L, N) for _ in range(4))
    da, e_da = new(K, N), new(K, N)
    carry, m_carry, e_carry = (new(B, K, N) for _ in range(3))
    for t in reversed(range(L)):
        A, e_A = decay(t)
        C, Bt, Gt, Du = c[:, t, None, :], b[:, t, None, :], G[:, t, :, None], (D * u)[:, t, :, None]
        e_Gt, e_Dt = e_G[:, t, :, None], e_D[:, t, :, None]
        cg = C * Gt
        g, m_g = cg + carry, cg.abs() + m_carry
        e_g = cg.abs() * e_Gt + e_carry + U * m_g + 2 * TINY
        carry, m_carry, e_carry = A * g, A * m_g, A * e_g + (e_A * A + FLUSHED) * m_g + 2 * TINY
        w, m_w = carry * h[t], m_carry * m[t]
        e_w = e_carry * m[t] + m_carry * e_h[t] + U * m_w + TINY
        db[:, t], dc[:, t] = (g * Du).sum(1), (h[t + 1] * Gt).sum(1)
        e_db[:, t] = (e_g * Du.abs() + m_g * Du.abs() * (e_Dt + U + by_k)).sum(1) + 2 * K * TINY
        e_dc[:, t] = (e_h[t + 1] * Gt.abs() + m[t + 1] * Gt.abs() * (e_Gt + by_k)).sum(1) + 2 * K * TINY
        gb, m_gb, wa, m_wa = (g * Bt).sum(-1), (m_g * Bt.abs()).sum(-1), (w * a).sum(-1), (m_w * a.abs()).sum(-1)
        e_gb, e_wa = (e_g * Bt.abs()).sum(-1) + (N + 2) * U * m_gb + 2 * N * TINY, (e_w * a.abs()).sum(-1) + (N + 6) * U * m_wa + 2 * N * TINY
        dG = skip * G[:, t]
        du[:, t] = dG + D[:, t] * gb
        e_du[:, t] = dG.abs() * (e_G[:, t] + 2 * U) + D[:, t] * (e_gb + m_gb * (e_D[:, t] + 3 * U)) + 4 * TINY
        sig = sigmoid(x[:, t])
        ddt[:, t] = (u[:, t] * gb + wa) * sig
        size_ddt[:, t] = (u[:, t].abs() * m_gb + m_wa) * sig
        e_ddt[:, t] = (u[:, t].abs() * e_gb + e_wa) * sig + size_ddt[:, t] * (e_sig[:, t] + 4 * U) + 4 * TINY
        da += (w * D[:, t, :, None]).sum(0)
        e_da += (e_w * D[:, t, :, None] + m_w * D[:, t, :, None] * (e_Dt + U + by_t)).sum(0) + 2 * B * TINY
    out |= dict(du=(du, e_du), ddt=(ddt, e_ddt), da=(da, e_da), db=(db, e_db), dc=(dc, e_dc))
    out["dd"] = None if d is None else ((G * u).sum((0, 1)), ((G * u).abs() * (e_G + U + by_t)).sum((0, 1)) + 2 * B * L * TINY)
    if z is None:
        out["dz"] = None
    else:
        f = sigmoid(z)
        size = f + (z * f * (1 - f)).abs()  # (its two terms cancel near z = -1.28)
        out["dz"] = dy * s * (f + z * f * (1 - f)), dy.abs() * size * (e_s + s_size * (6 * z.abs() + 14) * U) + 6 * TINY
    out["ddt_bias"] = None if dt_bias is None else (ddt.sum((0, 1)), (e_ddt + size_ddt * by_t).sum((0, 1)))
    return out


def within(got, want, error, dtype):
    """The largest part of what `got` may be off by that it is off by: at most 1.  One rounding to `dtype`, `error` (and a hundredth of it for products of
    errors), and half of the smallest step."""
    assert got.shape == want.shape
    got = got.double()
    half = torch.finfo(dtype).eps / 2 if dtype != torch.float32 else U
    info = torch.finfo(dtype)
    allowed = half * want.abs() + 1.01 * (1 + half) * error + info.smallest_normal * info.eps / 2
    part = ((got - want).abs() / allowed).max()
    return float(part) if torch.isfinite(got).all() else float("nan")
