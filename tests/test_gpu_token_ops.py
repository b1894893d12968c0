"""The operators between a block's linears against their definitions in 64 bits, where they can go wrong: one token, odd
widths and lengths, tile and chunk borders, each type, strided operands, both directions of time, states in and out."""
import pytest
import torch

import paper_2412_20386_amd as ptq
import token_ops_ref as ref

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TYPES = {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}
U = ref.U


def _near(got, want, magnitude, roundings, what):
    """Within the rounding to the result's type and `roundings` roundings of fp32 on the way."""
    got = got.detach().cpu().double()
    assert got.shape == want.shape, what
    half = torch.finfo(TYPES[what[0]]).eps / 2 if what[1] == "T" else U
    # (a subnormal fp16 result is off by half of its smallest step)
    tiny = torch.finfo(torch.float16).smallest_normal * torch.finfo(torch.float16).eps / 2
    off = (got - want).abs() - half * want.abs() - roundings * U * (1 + half) * magnitude - tiny
    assert torch.isfinite(got).all(), what
    assert off.max() <= 0, (what, float((got - want).abs().max()), float(off.max()))


class Draw:
    def __init__(self, seed):
        self.g = torch.Generator().manual_seed(seed)

    def __call__(self, *shape, scale=1.0, dtype=torch.float32):
        return (torch.randn(*shape, generator=self.g) * scale).to(dtype)


def _device(v, strided=0):
    """On the GPU; `strided`: as the last columns of a matrix that has as many more in front."""
    if v is None or not strided:
        return None if v is None else v.to(DEV)
    wide = torch.full((v.shape[0], v.shape[1] + strided), float("nan"), dtype=v.dtype, device=DEV)
    wide[:, strided:] = v.to(DEV)
    return wide[:, strided:]


def _time(v, B, L, reverse):
    v = v.double().view(B, L, -1)
    return v.flip(1) if reverse else v


def _guarded(rows, cols, dtype):
    """An output inside a larger buffer of a known pattern, and a check that nothing around it was written."""
    wide = torch.full((rows + 2, cols + 5), -7.0, dtype=dtype, device=DEV)

    def check():
        rest = wide.clone()
        rest[1:-1, 2:2 + cols] = -7.0
        assert (rest == -7.0).all()

    return wide[1:-1, 2:2 + cols], check


def _scan_inputs(seed, B, L, K, N, dtype, skip=True, gate=True, bias=True, state=False):
    n, T, M = Draw(seed), TYPES[dtype], B * L
    return dict(u=n(M, K, dtype=T), dt=n(M, K, scale=0.7, dtype=T), a=-torch.arange(1, N + 1, dtype=torch.float32) * torch.exp(n(K, N, scale=0.3)) * 0.5,
                b=n(M, N, dtype=T), c=n(M, N, dtype=T), d=n(K) if skip else None, z=n(M, K, dtype=T) if gate else None,
                dt_bias=n(K, scale=1.0) - 2 if bias else None), (n(B, K, N) if state else None)


BY_TOKEN = ("u", "dt", "b", "c", "z")
# B, L, K, N, type, reverse, state, strided, skip, gate, bias
SCANS = [
    (1, 1, 1, 1, "f32", False, False, 0, True, True, True),
    (1, 1, 16, 16, "f16", False, True, 0, True, True, True),
    (2, 15, 33, 16, "f16", False, True, 3, True, True, False),
    (2, 16, 64, 16, "bf16", True, False, 0, True, True, True),
    (3, 17, 40, 16, "f16", True, True, 0, False, False, True),
    (1, 31, 31, 4, "f32", False, True, 0, True, True, True),
    (1, 33, 7, 3, "f16", False, False, 1, True, True, True),
    (2, 50, 24, 5, "bf16", False, True, 5, True, False, True),
    (1, 64, 20, 17, "f16", True, True, 0, True, True, True),
    (2, 40, 19, 64, "f32", False, True, 0, True, True, True),
    (1, 65, 16, 33, "bf16", False, False, 2, True, True, True),
    (1, 197, 48, 16, "f16", False, True, 12, True, True, True),
    (1, 600, 18, 16, "f32", True, True, 0, True, True, True),
    (2, 1057, 5, 2, "f16", False, True, 0, True, True, True),
    (1, 9001, 3, 2, "f32", False, True, 0, True, True, True),     # as many chunks as there can be
    (1, 3000, 70, 16, "bf16", True, False, 0, True, True, True),
    (2, 256, 30, 11, "f16", False, True, 2, True, True, True),    # every tile of a sequence in one workgroup
    (5, 257, 20, 16, "f32", True, True, 0, True, True, True),
    (4100, 3, 64, 16, "f16", True, True, 0, True, True, True),    # a channel to a lane
    (4100, 10, 7, 13, "bf16", False, True, 3, True, True, True),
    (2, 70, 21, 32, "f16", False, True, 0, True, True, True),
    (3, 70, 16, 24, "bf16", True, False, 1, True, False, True),
    (40, 18, 1700, 7, "f16", False, True, 0, True, True, True),
    (1, 300, 33, 8, "f32", True, True, 0, True, True, True),
    (2050, 17, 66, 10, "f32", False, False, 0, False, True, True),
    (64, 3, 1030, 16, "f16", False, True, 0, True, True, True),   # two channels to a lane
    (70, 18, 992, 13, "bf16", True, False, 0, True, True, True),
]


@pytest.mark.parametrize("case", SCANS, ids=str)
def test_scan(case):
    B, L, K, N, dtype, reverse, with_state, strided, skip, gate, bias = case
    print("scan", case, flush=True)
    v, state = _scan_inputs(B * 1000 + L, B, L, K, N, dtype, skip, gate, bias, with_state)
    T, M = TYPES[dtype], B * L
    gpu = {k: _device(t, strided if k in BY_TOKEN else 0) for k, t in v.items()}
    y, untouched = _guarded(M, K, T)
    state_out = torch.empty((B, K, N), device=DEV)
    marks = torch.empty((ptq.scan_marks(L), B, K, N), device=DEV)
    first = _device(state)
    assert ptq.gated_scan(*gpu.values(), B, L, reverse=reverse, state=first, y=y, state_out=state_out, marks=marks) is y
    exact = {k: None if t is None else _time(t, B, L, reverse) if k in BY_TOKEN else t.double() for k, t in v.items()}
    state = None if state is None else state.double()
    (want, h, _), (size, h_size, _) = (ref.scan(**exact, state=state, magnitude=m) for m in (False, True))
    r = ref.scan_roundings(L, N)
    _near(_time(y.cpu(), B, L, reverse), want, size, r, (dtype, "T", "y"))
    untouched()
    _near(state_out, h[:, L], h_size[:, L], r, (dtype, "f32", "state_out"))
    _near(marks.transpose(0, 1), h[:, :L:8], h_size[:, :L:8], r, (dtype, "f32", "marks"))
    # without what is optional: the same bits
    assert torch.equal(ptq.gated_scan(*gpu.values(), B, L, reverse=reverse, state=first), y)

    # the backward pass
    dy = Draw(7)(M, K, dtype=T)
    outs = {n: _guarded(M, w, T) for n, w in (("du", K), ("ddt", K), ("db", N), ("dc", N), ("dz", K)) if n != "dz" or gate}
    grads = ptq.gated_scan_backward(_device(dy, strided), *gpu.values(), marks, B, L, reverse=reverse, **{n: o[0] for n, o in outs.items()})
    again = ptq.gated_scan_backward(_device(dy, strided), *gpu.values(), marks, B, L, reverse=reverse)
    want, size = (ref.scan_backward(_time(dy, B, L, reverse), **exact, state=state, magnitude=m) for m in (False, True))
    for name, got, other in zip(("du", "ddt", "da", "db", "dc", "dd", "dz", "ddt_bias"), grads, again):
        if want[name] is None:
            assert got is None and other is None
            continue
        assert torch.equal(got, other), name  # the same inputs: the same bits
        by_token = name in outs
        if by_token:
            outs[name][1]()
        # both passes' roundings, and the sums' over K, or over B and L
        _near(_time(got.cpu(), B, L, reverse) if by_token else got, want[name], size[name], 2 * r + (K if name in ("db", "dc") else B * L), (dtype, "T" if by_token else "f32", name))


@pytest.mark.parametrize("B,K,N,dtype,gate", [(1, 1, 1, "f32", True), (3, 50, 16, "f16", True), (2, 33, 5, "bf16", False), (5, 20, 64, "f16", True), (5, 20, 30, "bf16", True), (3, 30, 8, "f16", True), (2, 70, 3, "f32", True), (2, 9, 37, "bf16", True)])
def test_scan_step_by_step_is_the_scan(B, K, N, dtype, gate):
    """Token by token, in place, against the definition; and the step's own results against those of the scan over one token."""
    L, T = 9, TYPES[dtype]
    v, state = _scan_inputs(11, B, L, K, N, dtype, gate=gate, state=True)
    exact = {k: None if t is None else _time(t, B, L, False) if k in BY_TOKEN else t.double() for k, t in v.items()}
    (want, h, _), (size, h_size, _) = (ref.scan(**exact, state=state.double(), magnitude=m) for m in (False, True))
    now = state.to(DEV)
    for t in range(L):
        one = {k: None if x is None else (x.view(B, L, -1)[:, t].to(DEV) if k in BY_TOKEN else x.to(DEV)) for k, x in v.items()}
        kept, after = now.clone(), torch.full_like(now, -7.0)
        other = ptq.gated_scan_step(*one.values(), now, state_out=after)
        assert torch.equal(now, kept)
        y = ptq.gated_scan_step(*one.values(), now)
        assert torch.equal(y, other) and torch.equal(now, after)
        _near(y, want[:, t], size[:, t], ref.scan_roundings(t + 1, N), (dtype, "T", f"y {t}"))
        _near(now, h[:, t + 1], h_size[:, t + 1], ref.scan_roundings(t + 1, N), (dtype, "f32", f"state {t}"))
    assert y.dtype == T


def test_scan_in_segments_is_the_scan():
    """A sequence in three calls that hand the state on."""
    B, K, N, L = 2, 40, 16, 150
    v, _ = _scan_inputs(5, B, L, K, N, "f32")
    gpu = {k: t.to(DEV) for k, t in v.items()}
    whole = torch.empty((B, K, N), device=DEV)
    y = ptq.gated_scan(*gpu.values(), B, L, state_out=whole).view(B, L, K)
    state, parts, at = None, [], 0
    for n in (1, 100, 49):
        part = {k: (t.view(B, L, -1)[:, at:at + n].reshape(B * n, -1) if k in BY_TOKEN else t) for k, t in gpu.items()}
        after = torch.empty((B, K, N), device=DEV)
        parts.append(ptq.gated_scan(*part.values(), B, n, state=state, state_out=after).view(B, n, K))
        state, at = after, at + n
    exact = {k: _time(t, B, L, False) if k in BY_TOKEN else t.double() for k, t in v.items()}
    size, h_size, _ = ref.scan(**exact, magnitude=True)
    r = 2 * ref.scan_roundings(L, N)
    _near(torch.cat(parts, 1), y.cpu().double(), size, r, ("f32", "T", "y"))
    _near(state, whole.cpu().double(), h_size[:, L], r, ("f32", "f32", "state"))


def test_scan_far_steps_and_infinities():
    """Steps of 50 forget everything, steps of 1e-6 keep everything, an infinite step lets nothing through but the token itself; an infinite
    or NaN input stays in its channel."""
    B, L, K, N = 1, 40, 32, 16
    v, _ = _scan_inputs(6, B, L, K, N, "f32", bias=False, gate=False)
    v["dt"][:, 0], v["dt"][:, 1] = 50.0, -14.0
    v["dt"][5, 2], v["u"][7, 3], v["u"][9, 4] = float("inf"), float("inf"), float("nan")
    gpu = {k: None if t is None else t.to(DEV) for k, t in v.items()}
    y = ptq.gated_scan(*gpu.values(), B, L).cpu().double()
    exact = {k: None if t is None else _time(t, B, L, False) if k in BY_TOKEN else t.double() for k, t in v.items()}
    (want, _, _), (size, _, _) = (ref.scan(**exact, magnitude=m) for m in (False, True))
    fine = [k for k in range(K) if k not in (2, 3, 4)]
    _near(y[:, fine], want[0][:, fine], size[0][:, fine], ref.scan_roundings(L, N), ("f32", "T", "y"))
    for k, t in ((2, 5), (3, 7), (4, 9)):
        _near(y[:t, k], want[0][:t, k], size[0][:t, k], ref.scan_roundings(L, N), ("f32", "T", "y"))
        assert not torch.isfinite(y[t:, k]).all()


# B, L, K, W, type, silu, reverse, state, strided, bias
CONVS = [
    (1, 1, 1, 2, "f32", True, False, False, 0, True),
    (1, 1, 8, 4, "f16", True, False, True, 0, True),
    (2, 2, 9, 4, "f16", True, True, True, 0, True),
    (3, 3, 16, 3, "bf16", False, False, False, 3, True),
    (2, 4, 100, 4, "f16", True, False, True, 100, False),
    (2, 5, 65, 2, "f32", True, True, True, 1, True),
    (1, 197, 384, 4, "f16", True, False, False, 384, True),
    (5, 33, 520, 3, "bf16", True, True, True, 0, True),
    (64, 50, 300, 4, "f16", True, False, True, 0, True),
    (2, 3000, 17, 4, "f32", True, False, True, 0, True),
]


@pytest.mark.parametrize("case", CONVS, ids=str)
def test_conv(case):
    B, L, K, W, dtype, silu, reverse, with_state, strided, with_bias = case
    print("conv", case, flush=True)
    n, T, M = Draw(L * 7 + K), TYPES[dtype], B * L
    x, w, bias = n(M, K, dtype=T), n(K, W), n(K) if with_bias else None
    state = n(B, W - 1, K, dtype=T) if with_state else None
    y, untouched = _guarded(M, K, T)
    after = torch.empty((B, W - 1, K), dtype=T, device=DEV)
    gx, gw, gb, gs = _device(x, strided), w.to(DEV), _device(bias), _device(state)
    ptq.token_conv(gx, gw, gb, B, L, silu=silu, reverse=reverse, state=gs, y=y, state_out=after)
    ex, es = _time(x, B, L, reverse), None if state is None else state.double()
    eb = None if bias is None else bias.double()
    (want, last), (size, _) = (ref.conv(ex, w.double(), eb, es, silu, magnitude=m) for m in (False, True))
    # W products and their sum, the bias, and the activation (8, and the exponent's 2 |p| e^-|p| times: below 1.1 in all)
    _near(_time(y.cpu(), B, L, reverse), want, 1.1 * size, W + 12, (dtype, "T", "y"))
    untouched()
    assert torch.equal(after.cpu().double(), last)

    dy = n(M, K, dtype=T)
    dx, untouched = _guarded(M, K, T)
    grads = ptq.token_conv_backward(_device(dy, strided), gx, gw, gb, B, L, silu=silu, reverse=reverse, state=gs, dx=dx)
    again = ptq.token_conv_backward(_device(dy, strided), gx, gw, gb, B, L, silu=silu, reverse=reverse, state=gs)
    untouched()
    edy = _time(dy, B, L, reverse)
    want, size = (ref.conv_backward(edy, ex, w.double(), eb, es, silu, magnitude=m) for m in (False, True))
    # the derivative: its own 16 roundings, and those of p (W + 1 of its terms' magnitudes), of which it takes half at most
    p_size = ref.conv(ex, w.double(), eb, es, silu, magnitude=True)[0].max() if silu else 0.0
    extra = (W + 1) * p_size / 2 + 16
    for name, got, other in zip(("dx", "dw", "dbias"), grads, again):
        if want[name] is None:
            assert got is None
            continue
        assert torch.equal(got, other), name
        by_token = name == "dx"
        _near(_time(got.cpu(), B, L, reverse) if by_token else got, want[name], 1.1 * size[name], extra + (W + 1 if by_token else B * L), (dtype, "T" if by_token else "f32", name))


@pytest.mark.parametrize("B,K,W,dtype", [(1, 1, 2, "f32"), (3, 50, 4, "f16"), (16, 768, 4, "bf16"), (4, 30, 3, "f16")])
def test_conv_step_by_step_is_the_conv(B, K, W, dtype):
    n, T, L = Draw(K), TYPES[dtype], 6
    x, w, bias, state = n(B, L, K, dtype=T).to(DEV), n(K, W).to(DEV), n(K).to(DEV), n(B, W - 1, K, dtype=T).to(DEV)
    after = torch.empty_like(state)
    y = ptq.token_conv(x.view(B * L, K), w, bias, B, L, state=state, state_out=after).view(B, L, K)
    now = state.clone()
    for t in range(L):
        kept, out = now.clone(), torch.empty_like(now)
        other = ptq.token_conv_step(x[:, t], w, bias, now, state_out=out)
        assert torch.equal(now, kept)
        assert torch.equal(ptq.token_conv_step(x[:, t], w, bias, now), y[:, t])  # the same sums: the same bits
        assert torch.equal(other, y[:, t]) and torch.equal(out, now)
    assert torch.equal(now, after)


# M, K, type, stream, residual, G, post, scale, strided
NORMS = [
    (1, 1, "f32", "f32", True, None, False, 1.0, 0),
    (1, 8, "f16", "f16", True, 1, True, 0.5, 0),
    (7, 1001, "f16", "f32", True, 7, True, 1.0, 5),
    (6, 384, "bf16", "bf16", True, 2, True, 0.875, 0),
    (300, 192, "f16", "f16", True, 1, False, 1.0, 0),
    (300, 192, "f16", "f32", False, 100, True, 1.0, 3),
    (5000, 24, "f32", "f32", True, 5000, True, 1.0, 0),
    (2100, 768, "bf16", "f32", True, 3, True, 1.0, 0),
    (9, 1025, "f16", "f16", True, None, True, 1.0, 1),
    (12, 4096, "bf16", "bf16", True, 4, True, 1.0, 0),
    (10, 4097, "f16", "f32", True, 10, False, 1.0, 0),
    (3, 16384, "f16", "f32", True, 1, True, 1.0, 0),
    (4, 10007, "f32", "f32", False, None, False, 1.0, 1),
]


@pytest.mark.parametrize("case", NORMS, ids=str)
def test_norm(case):
    M, K, dtype, stream, with_residual, G, post, scale, strided = case
    print("norm", case, flush=True)
    n, T, S = Draw(M + K), TYPES[dtype], TYPES[stream]
    h, residual = n(M, K, dtype=T), n(M, K, scale=2.0, dtype=S) if with_residual else None
    w, gate, w_post = n(K) + 1.5, (n(G, K) + 1 if G else None), (n(K) + 1.5 if post else None)
    y, y_untouched = _guarded(M, K, T)
    r, r_untouched = _guarded(M, K, S)
    params = [_device(t) for t in (w, gate, w_post)]
    gh = _device(h, strided)
    out = ptq.residual_norm(gh, _device(residual, strided), *params, scale=scale, eps=1e-5, y=y, residual_out=r)
    assert out[0] is y and out[1] is r
    y_untouched(), r_untouched()
    d = lambda t: None if t is None else t.double()  # noqa: E731
    want_y, want_r = ref.residual_norm(d(h), d(residual), d(w), d(gate), d(w_post), scale)
    # a norm: the sum of squares (a square root halves its K + 3), mean and root (6), two products; r: a product and a sum more
    f = K / 2 + 12
    size = (d(h).abs() if w_post is None else ref.norm(d(h), 1e-5).abs() * d(w_post).abs()) * (1.0 if gate is None else ref.rows_of_gate(d(gate), M).abs())
    size = size + (0 if residual is None else abs(scale) * d(residual).abs())
    _near(r, want_r, size, f, (stream, "T", "r"))
    rms = torch.sqrt(want_r.square().mean(-1, keepdim=True) + 1e-5)
    # an error of r, f U size, moves y by that over rms(r), and rms(r) by at most the root of its mean square
    y_size = size / rms * d(w).abs() + want_y.abs() * (1 + (size / rms).square().mean(-1, keepdim=True).sqrt())
    _near(y, want_y, y_size, 2 * f, (dtype, "T", "y"))

    for with_dr in (True, False):
        dy, dr = n(M, K, dtype=T), n(M, K, dtype=S) if with_dr else None
        dh, dh_untouched = _guarded(M, K, T)
        dres, dres_untouched = _guarded(M, K, S)
        outs = dict(dh=dh) if residual is None else dict(dh=dh, dresidual=dres)
        args = (_device(dy, strided), _device(dr, strided), gh, r, *params)
        grads = ptq.residual_norm_backward(*args, scale=scale, eps=1e-5, first=residual is None, **outs)
        again = ptq.residual_norm_backward(*args, scale=scale, eps=1e-5, first=residual is None)
        dh_untouched(), dres_untouched()
        er = r.cpu().double()
        want = ref.residual_norm_backward(d(dy), d(dr), d(h), er, d(w), d(gate), d(w_post), scale)
        # magnitudes: every norm's gradient is rms^-1 (t - n mean(t n)), its terms t and |n| mean |t n|
        def through(t, v):
            inverse = 1 / torch.sqrt(v.square().mean(-1, keepdim=True) + 1e-5)
            return inverse * (t + v.abs() * inverse * (t * v.abs() * inverse).mean(-1, keepdim=True))
        e = through((d(dy) * d(w)).abs(), er) + (0 if dr is None else d(dr).abs())
        fe = e * (1.0 if gate is None else ref.rows_of_gate(d(gate), M).abs())
        q = d(h).abs() if w_post is None else ref.norm(d(h), 1e-5).abs() * d(w_post).abs()
        size = dict(dh=fe if w_post is None else through(fe * d(w_post).abs(), d(h)), dresidual=abs(scale) * e, dw=(d(dy) * ref.norm(er, 1e-5)).abs().sum(0),
                    dgate=None if gate is None else (e * q).view(gate.shape[0], -1, K).sum(1), dw_post=None if w_post is None else (fe * ref.norm(d(h), 1e-5).abs()).sum(0))
        for name, got, other in zip(("dh", "dresidual", "dw", "dgate", "dw_post"), grads, again):
            if want[name] is None or (name == "dresidual" and residual is None):
                assert got is None, name
                continue
            assert torch.equal(got, other), name
            # both norms' roots and means: four sums over K; the parameters' sums over M rows
            _near(got, want[name], size[name], 2 * f + 2 * K + 24 + (M if name in ("dw", "dgate", "dw_post") else 0),
                  ({"dh": dtype, "dresidual": stream}.get(name, "f32"), "T", name))


def test_no_sequences():
    """Nothing to do, and gradients of parameters that are zero."""
    e = lambda *s: torch.empty(s, device=DEV)  # noqa: E731
    a, w, ones = e(8, 4), e(8, 3), torch.ones(8, device=DEV)
    assert ptq.gated_scan(e(0, 8), e(0, 8), a, e(0, 4), e(0, 4), None, None, None, 0, 5).shape == (0, 8)
    grads = ptq.gated_scan_backward(e(0, 8), e(0, 8), e(0, 8), a, e(0, 4), e(0, 4), ones, None, ones, e(1, 0, 8, 4), 0, 5)
    assert all((grads[i] == 0).all() for i in (2, 5, 7)) and grads[2].shape == (8, 4)
    assert ptq.gated_scan_step(e(0, 8), e(0, 8), a, e(0, 4), e(0, 4), None, None, None, e(0, 8, 4)).shape == (0, 8)
    assert ptq.token_conv(e(0, 8), w, None, 0, 5).shape == (0, 8)
    assert all((g == 0).all() for g in ptq.token_conv_backward(e(0, 8), e(0, 8), w, ones, 0, 5)[1:])
    assert ptq.residual_norm(e(0, 8), e(0, 8), ones)[0].shape == (0, 8)
    assert all((g == 0).all() for g in ptq.residual_norm_backward(e(0, 8), None, e(0, 8), e(0, 8), ones, e(2, 8), ones)[2:])


def test_rows_of_zeros():
    """A row of zeros has a norm of zeros and finite gradients."""
    h = torch.zeros(3, 40, device=DEV)
    w = torch.ones(40, device=DEV)
    y, r = ptq.residual_norm(h, h, w, None, w)
    assert (y == 0).all() and (r == 0).all()
    assert all(torch.isfinite(g).all() for g in ptq.residual_norm_backward(torch.ones_like(h), None, h, r, w, None, w) if g is not None)
