"""The operators as a block uses them: among the library's linears, on the columns and halves that those leave, in both directions of
time, step by step, on a stream of the caller's and in a captured graph; and on matrices of more than 2^31 elements."""
import pytest
import torch

import paper_2412_20386_amd as ptq
import token_ops_ref as ref
from test_gpu_token_ops import _near

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
H = torch.float16
B, L, DIM, K, N, R, W = 3, 37, 48, 96, 16, 8, 4
M = B * L


def _weights(seed):
    g = torch.Generator().manual_seed(seed)
    n = lambda *s, scale=1.0, t=torch.float32: (torch.randn(*s, generator=g) * scale).to(t).to(DEV)  # noqa: E731
    side = lambda: dict(conv=n(K, W, scale=0.5), conv_bias=n(K, scale=0.1), x_proj=n(R + 2 * N, K, scale=0.1, t=H), dt_proj=n(K, R, scale=0.3, t=H),  # noqa: E731
                        dt_bias=n(K) - 3, a=-torch.arange(1, N + 1, device=DEV, dtype=torch.float32) * torch.exp(n(K, N, scale=0.2)), d=n(K))
    return dict(norm=n(DIM, scale=0.1) + 1, post=n(DIM, scale=0.1) + 1, gate=n(B, DIM), in_proj=n(2 * K, DIM, scale=0.15, t=H), out_proj=n(DIM, K, scale=0.1, t=H),
                sides=(side(), side())), n(M, DIM, t=H), n(M, DIM)


def _block(w, h, stream):
    """The norms, then a block that scans its tokens both ways: (output, stream behind it, everything on the way)."""
    y, r = ptq.residual_norm(h, stream, w["norm"], w["gate"], w["post"], scale=0.9)
    xz = ptq.f16_linear(y, w["in_proj"], None)
    kept, outs = [], []
    for reverse, s in zip((False, True), w["sides"]):
        u = ptq.token_conv(xz[:, :K], s["conv"], s["conv_bias"], B, L, reverse=reverse)
        dbc = ptq.f16_linear(u, s["x_proj"], None)
        dt = ptq.f16_linear(dbc[:, :R], s["dt_proj"], None)
        marks = torch.empty((ptq.scan_marks(L), B, K, N), device=DEV)
        out = ptq.gated_scan(u, dt, s["a"], dbc[:, R:R + N], dbc[:, R + N:], s["d"], xz[:, K:], s["dt_bias"], B, L, reverse=reverse, marks=marks)
        kept.append((u, dbc, dt, marks, out))
        outs.append(out)
    return ptq.f16_linear(outs[0] + outs[1], w["out_proj"], None), r, (y, xz, kept)


def _backward(w, h, r, way, dout, dr):
    """Gradients of the block's operators, those of the linears by torch's products."""
    y, xz, kept = way
    dsum = dout @ w["out_proj"]
    dxz, grads = torch.zeros_like(xz), []
    for reverse, s, (u, dbc, dt, marks, _) in zip((False, True), w["sides"], kept):
        d_dbc = torch.empty_like(dbc)
        dz = torch.empty_like(u)
        du, ddt, da, _, _, dd, _, dbias = ptq.gated_scan_backward(dsum, u, dt, s["a"], dbc[:, R:R + N], dbc[:, R + N:], s["d"], xz[:, K:], s["dt_bias"], marks, B, L,
                                                                 reverse=reverse, db=d_dbc[:, R:R + N], dc=d_dbc[:, R + N:], dz=dz)
        d_dbc[:, :R] = ddt @ s["dt_proj"]
        du = du + d_dbc @ s["x_proj"]
        dx, dw, dcb = ptq.token_conv_backward(du, xz[:, :K], s["conv"], s["conv_bias"], B, L, reverse=reverse)
        dxz[:, :K] += dx
        dxz[:, K:] += dz
        grads += [du, ddt, da, d_dbc, dd, dbias, dx, dw, dcb, dz]
    dy = dxz @ w["in_proj"]
    return grads + list(ptq.residual_norm_backward(dy, dr, h, r, w["norm"], w["gate"], w["post"], scale=0.9)) + [dy]


def _time(v, reverse):
    v = v.detach().cpu().double().view(B, L, -1)
    return v.flip(1) if reverse else v


def test_a_block_stage_by_stage():
    """Each operator's results from the very inputs that it got in the block."""
    w, h, stream = _weights(1)
    d = lambda t: t.detach().cpu().double()  # noqa: E731
    out, r, (y, xz, kept) = _block(w, h, stream)
    want_y, want_r = ref.residual_norm(d(h), d(stream), d(w["norm"]), d(w["gate"]), d(w["post"]), 0.9)
    # the norms: K / 2 + 12 roundings of the terms of r, and of y through r (terms up to 4 times y's size here)
    size = ref.norm(d(h), 1e-5).abs() * d(w["post"]).abs() * ref.rows_of_gate(d(w["gate"]), M).abs() + 0.9 * d(stream).abs()
    _near(r, want_r, size, DIM / 2 + 12, ("f32", "T", "r"))
    rms = torch.sqrt(want_r.square().mean(-1, keepdim=True) + 1e-5)
    _near(y, want_y, size / rms * d(w["norm"]).abs() + want_y.abs() * (1 + (size / rms).square().mean(-1, keepdim=True).sqrt()), DIM + 24, ("f16", "T", "y"))
    for reverse, s, (u, dbc, dt, marks, o) in zip((False, True), w["sides"], kept):
        x = _time(xz[:, :K], reverse)
        want, size = (ref.conv(x, d(s["conv"]), d(s["conv_bias"]), magnitude=m)[0] for m in (False, True))
        _near(_time(u, reverse), want, 1.1 * size, W + 12, ("f16", "T", "u"))
        args = dict(u=_time(u, reverse), dt=_time(dt, reverse), a=d(s["a"]), b=_time(dbc[:, R:R + N], reverse), c=_time(dbc[:, R + N:], reverse), d=d(s["d"]),
                    z=_time(xz[:, K:], reverse), dt_bias=d(s["dt_bias"]))
        want, size = (ref.scan(**args, magnitude=m)[0] for m in (False, True))
        _near(_time(o, reverse), want, size, ref.scan_roundings(L, N), ("f16", "T", "o"))
    assert torch.isfinite(out).all()
    # serving the same tokens one by one in the first direction: the states go from step to step
    s, (u, dbc, dt, _, o) = w["sides"][0], kept[0]
    conv_state, state = torch.zeros((B, W - 1, K), dtype=H, device=DEV), torch.zeros((B, K, N), device=DEV)
    at = lambda v, t: v.view(B, L, -1)[:, t] if v.is_contiguous() else v[t::L]  # noqa: E731
    got = []
    for t in range(L):
        u_t = ptq.token_conv_step(at(xz[:, :K], t), s["conv"], s["conv_bias"], conv_state)
        assert torch.equal(u_t, at(u, t))
        got.append(ptq.gated_scan_step(u_t, at(dt, t), s["a"], at(dbc[:, R:R + N], t), at(dbc[:, R + N:], t), s["d"], at(xz[:, K:], t), s["dt_bias"], state))
    args = {k: (v if k in ("a", "d", "dt_bias") else v) for k, v in args.items()}
    args = dict(u=_time(u, 0), dt=_time(dt, 0), a=d(s["a"]), b=_time(dbc[:, R:R + N], 0), c=_time(dbc[:, R + N:], 0), d=d(s["d"]), z=_time(xz[:, K:], 0), dt_bias=d(s["dt_bias"]))
    want, size = (ref.scan(**args, magnitude=m)[0] for m in (False, True))
    _near(torch.stack(got, 1), want, size, ref.scan_roundings(L, N), ("f16", "T", "steps"))


def test_with_the_quantized_linears():
    """The scan's output through the quantizer and the W8A8 linear, the norm's through the dynamic one: what they read is what was written."""
    w, h, stream = _weights(2)
    _, _, (y, xz, kept) = _block(w, h, stream)
    wq, s_w, inv_m = ptq.fold_smoothing(w["out_proj"], torch.ones(K, device=DEV))
    s_tok = torch.full((L,), 0.02, device=DEV)
    o = kept[0][4]
    out = ptq.w8a8_linear(ptq.quantize_pts(o, inv_m, s_tok, B, L), wq, s_tok, s_w, None, B, L)
    codes = torch.clamp(torch.round(o.float() / 0.02), -127, 127)
    assert (out.float() - codes @ (wq.float() * s_w[:, None]).t() * 0.02).abs().max() < 0.02
    xq, steps = ptq.quantize_dynamic(y, None)
    assert (xq.float() * steps[:, None] - y.float()).abs().max() <= 0.51 * steps.max()


def test_on_another_stream_and_in_a_graph():
    """Forward and backward captured into a graph: replays with new inputs give the eager bits, eager work and another graph between them."""
    w, h, stream = _weights(3)
    g = torch.Generator(device=DEV).manual_seed(9)
    n = lambda *s, t=H: torch.randn(*s, generator=g, device=DEV).to(t)  # noqa: E731
    dout, dr = n(M, DIM), n(M, DIM, t=torch.float32)

    def run():
        out, r, way = _block(w, h, stream)
        return [out, r, *_backward(w, h, r, way, dout, dr)]

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    eager = [t.clone() for t in run()]
    with torch.cuda.stream(side):
        other = run()
    side.synchronize()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(eager, other))
    graphs = []
    for _ in range(2):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            outs = run()
        graphs.append((graph, outs))
    for rep in range(4):
        for t in (h, stream, dout, dr):
            t.copy_(n(*t.shape, t=t.dtype))
        want = [t.clone() for t in run()]
        torch.cuda.synchronize()
        for graph, outs in graphs:
            graph.replay()
        torch.cuda.synchronize()
        for _, outs in graphs:
            for i, (a, b) in enumerate(zip(want, outs)):
                assert torch.equal(a, b), (rep, i)


def test_long_sequences_in_a_graph():
    """Chunks and their workspaces: two graphs of different lengths replayed in turn."""
    graphs = []
    side = torch.cuda.Stream()
    for length in (700, 2500):
        g = torch.Generator(device=DEV).manual_seed(length)
        n = lambda *s: torch.randn(*s, generator=g, device=DEV)  # noqa: E731
        v = [n(length, K), n(length, K), -torch.rand(K, N, generator=g, device=DEV) * 4, n(length, N), n(length, N), n(K), n(length, K), n(K) - 2]
        dy, marks = n(length, K), torch.empty((ptq.scan_marks(length), 1, K, N), device=DEV)

        def run(v=v, dy=dy, marks=marks, length=length):
            y = ptq.gated_scan(*v, 1, length, marks=marks)
            return [y, *ptq.gated_scan_backward(dy, *v, marks, 1, length)]

        want = [t.clone() for t in run()]
        graph = torch.cuda.CUDAGraph()
        torch.cuda.synchronize()
        with torch.cuda.graph(graph, stream=side):
            outs = run()
        graphs.append((graph, outs, want))
    for _ in range(3):
        for graph, outs, want in graphs:
            graph.replay()
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(outs, want))


def test_states_are_not_read_and_written_at_once():
    """Where several workgroups share a sequence, state_out may not be state."""
    state = torch.zeros((1, 16, 16), device=DEV)
    m = torch.zeros((5, 16), dtype=H, device=DEV)
    with pytest.raises(ValueError, match="not the buffer of state"):
        ptq.gated_scan(m, m, state[0], m, m, None, None, None, 1, 5, state=state, state_out=state)
    state = torch.zeros((1, 3, 16), dtype=H, device=DEV)
    with pytest.raises(ValueError, match="not the buffer of state"):
        ptq.token_conv(m, torch.zeros((16, 4), device=DEV), None, 1, 5, state=state, state_out=state)


def test_offsets_beyond_32_bits():
    """The last rows of matrices with more than 2^31 elements: the same results as those of a dense copy of them."""
    rows, pitch, k, n = 70000, 40000, 24, 4
    big = torch.empty((rows, pitch), dtype=H, device=DEV)  # 5.6 GB
    g = torch.Generator(device=DEV).manual_seed(1)
    dense = torch.randn(rows, k, generator=g, device=DEV).to(H)
    big[:, :k] = dense
    out = big[:, 100:100 + k]
    f = lambda *s: torch.randn(*s, generator=g, device=DEV)  # noqa: E731
    a, b, w = -torch.rand(k, n, generator=g, device=DEV), f(rows, n).to(H), f(k, 4)
    for batch, length in ((1, rows), (rows, 1), (700, 100)):
        want = ptq.gated_scan(dense, dense, a, b, b, None, dense, None, batch, length)
        assert torch.equal(ptq.gated_scan(big[:, :k], big[:, :k], a, b, b, None, big[:, :k], None, batch, length, y=out), want)
        want = ptq.token_conv(dense, w, None, batch, length)
        assert torch.equal(ptq.token_conv(big[:, :k], w, None, batch, length, y=out), want)
        want = ptq.token_conv_backward(dense, dense, w, None, batch, length)
        got = ptq.token_conv_backward(big[:, :k], big[:, :k], w, None, batch, length, dx=out)
        assert all(torch.equal(x, y) for x, y in zip(got[:2], want[:2]))
    want, _ = ptq.residual_norm(dense, dense, w[:, 0].contiguous())
    got, _ = ptq.residual_norm(big[:, :k], big[:, :k], w[:, 0].contiguous(), y=out, residual_out=big[:, 200:200 + k])
    assert torch.equal(got, want)
    marks = torch.empty((ptq.scan_marks(rows), 1, k, n), device=DEV)
    ptq.gated_scan(dense, dense, a, b, b, None, dense, None, 1, rows, marks=marks)
    want = ptq.gated_scan_backward(dense, dense, dense, a, b, b, None, dense, None, marks, 1, rows)
    x = big[:, :k]
    got = ptq.gated_scan_backward(x, x, x, a, b, b, None, x, None, marks, 1, rows, du=out, ddt=big[:, 200:200 + k], dz=big[:, 300:300 + k])
    assert all((x is None and y is None) or torch.equal(x, y) for x, y in zip(got, want))
