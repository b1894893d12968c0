"""The operators between a block's linears in 64 bits, from their definitions, and how far a result in 32 bits may be off.

Every function takes torch tensors on the CPU, in the order of time ([B, L, X]), and computes in float64.  `magnitude`
replaces every term of every sum by its absolute value: a sum of n terms in fp32, each computed with c roundings, is within
(n + c) 2^-24 of the sum of their magnitudes, and what a result is computed from passes that error on in the same proportion.
"""
import torch

U = 2.0 ** -24  # half a step of fp32: one rounding


def sigmoid(v):
    return 1.0 / (1.0 + torch.exp(-v))


def softplus(v):
    return torch.clamp(v, min=0) + torch.log1p(torch.exp(-v.abs()))


def scan(u, dt, a, b, c, d, z, dt_bias, state=None, magnitude=False):
    """(y, states [B, L + 1, K, N] from the one before the first token on, s)"""
    f = torch.abs if magnitude else (lambda v: v)
    B, L, K = u.shape
    D = softplus(dt + (0 if dt_bias is None else dt_bias))
    h = [torch.zeros(B, K, a.shape[1], dtype=torch.float64) if state is None else f(state)]
    for t in range(L):
        h.append(torch.exp(D[:, t, :, None] * a) * h[-1] + (D * f(u))[:, t, :, None] * f(b)[:, t, None, :])
    h = torch.stack(h, 1)
    s = (h[:, 1:] * f(c)[:, :, None, :]).sum(-1) + (0 if d is None else f(d) * f(u))
    return (s if z is None else s * f(z * sigmoid(z))), h, s


def scan_backward(dy, u, dt, a, b, c, d, z, dt_bias, state=None, magnitude=False):
    f = torch.abs if magnitude else (lambda v: v)
    B, L, K = u.shape
    x = dt + (0 if dt_bias is None else dt_bias)
    D = softplus(x)
    _, h, s = scan(u, dt, a, b, c, d, z, dt_bias, state, magnitude)
    G, dz = f(dy), None
    if z is not None:
        G = f(dy) * f(z * sigmoid(z))
        # the gate's derivative is a sum of sigma(z) and z sigma(z) (1 - sigma(z)), which cancel near z = -1.28: each term is rounded in
        # proportion to itself, so the error there is that of the terms, not of their difference
        dz = f(dy) * s * (sigmoid(z) + f(z * sigmoid(z) * (1 - sigmoid(z))))
    e = torch.exp(D[..., None] * a)
    g, carry = torch.zeros_like(h[:, 1:]), torch.zeros_like(h[:, 0])
    for t in reversed(range(L)):
        g[:, t] = f(c)[:, t, None, :] * G[:, t, :, None] + carry
        carry = e[:, t] * g[:, t]
    w = g * e * h[:, :-1]
    gb = (g * f(b)[:, :, None, :]).sum(-1)
    dD = f(u) * gb + (w * f(a)).sum(-1)
    ddt = dD * sigmoid(x)
    return dict(du=(0 if d is None else f(d) * G) + D * gb, ddt=ddt, da=(w * D[..., None]).sum((0, 1)), db=(g * (D * f(u))[..., None]).sum(2),
                dc=(h[:, 1:] * G[..., None]).sum(2), dd=None if d is None else (G * f(u)).sum((0, 1)), dz=dz,
                ddt_bias=None if dt_bias is None else ddt.sum((0, 1)))


def scan_roundings(L, N):
    """Roundings that a state passes through: for each step those of D (8: softplus), of the exponent (2, which count |D a| <=
    e^|D a| times), of the exponential (2), of D u b (2) and of the multiply-add (1); then N products and their sum, the skip, and the
    gate (10)."""
    return 15 * L + 2 * N + 24


def conv(x, w, bias, state=None, silu=True, magnitude=False):
    f = torch.abs if magnitude else (lambda v: v)
    B, L, K = x.shape
    W = w.shape[1]
    before = torch.zeros(B, W - 1, K, dtype=torch.float64) if state is None else state
    full = f(torch.cat([before, x], 1))
    p = sum(full[:, j:j + L] * f(w)[:, j] for j in range(W)) + (0 if bias is None else f(bias))
    return (p * sigmoid(p) if silu and not magnitude else p), torch.cat([before, x], 1)[:, L:]


def conv_backward(dy, x, w, bias, state=None, silu=True, magnitude=False):
    f = torch.abs if magnitude else (lambda v: v)
    B, L, K = x.shape
    W = w.shape[1]
    before = torch.zeros(B, W - 1, K, dtype=torch.float64) if state is None else state
    full = torch.cat([before, x], 1)
    dp = f(dy)
    if silu and not magnitude:  # (the derivative is below 1.1)
        p = sum(full[:, j:j + L] * w[:, j] for j in range(W)) + (0 if bias is None else bias)
        dp = dy * sigmoid(p) * (1 + p * (1 - sigmoid(p)))
    late = torch.cat([dp, torch.zeros(B, W - 1, K, dtype=torch.float64)], 1)
    dx = sum(late[:, W - 1 - j:W - 1 - j + L] * f(w)[:, j] for j in range(W))
    dw = torch.stack([(dp * f(full)[:, j:j + L]).sum((0, 1)) for j in range(W)], 1)
    return dict(dx=dx, dw=dw, dbias=None if bias is None else dp.sum((0, 1)))


def norm(v, eps):
    return v / torch.sqrt(v.square().mean(-1, keepdim=True) + eps)


def rows_of_gate(gate, M):
    return 1.0 if gate is None else gate.repeat_interleave(M // gate.shape[0], 0)


def residual_norm(h, residual, w, gate=None, w_post=None, scale=1.0, eps=1e-5):
    q = h if w_post is None else norm(h, eps) * w_post
    r = rows_of_gate(gate, h.shape[0]) * q + (0 if residual is None else scale * residual)
    return norm(r, eps) * w, r


def residual_norm_backward(dy, dr, h, r, w, gate=None, w_post=None, scale=1.0, eps=1e-5):
    """The gradients by their formulas, r being what the forward pass left (rounded to the stream's type)."""
    def through(t, v):
        inverse = 1 / torch.sqrt(v.square().mean(-1, keepdim=True) + eps)
        return inverse * (t - v * inverse * (t * v * inverse).mean(-1, keepdim=True))

    e = through(dy * w, r) + (0 if dr is None else dr)
    f = rows_of_gate(gate, h.shape[0]) * e
    q = h if w_post is None else norm(h, eps) * w_post
    return dict(dh=f if w_post is None else through(f * w_post, h), dresidual=scale * e, dw=(dy * norm(r, eps)).sum(0),
                dgate=None if gate is None else (e * q).view(gate.shape[0], -1, h.shape[1]).sum(1), dw_post=None if w_post is None else (f * norm(h, eps)).sum(0))
