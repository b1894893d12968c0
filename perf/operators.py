"""The operators between the linears of a Mamba block, and how they are measured.

Every case is one pass through one operator, forward, in training (forward and backward, or the backward pass alone where
the forward's outputs are among its inputs), or for one token per sequence:

  scan, scan_train, scan_step    the gated linear recurrence between dt_proj and out_proj
  conv, conv_train, conv_step    the short convolution over tokens between in_proj and x_proj
  norm, norm_train               the norms after and before a block with its gate and the residual stream

Matrices are token-major, [B * L, K].  K is the width, N the number of states per channel, W the taps of the convolution.
`strided` cases read their operands where a block has them: the halves of in_proj's output and the columns of x_proj's.

`own` false computes them in elementary operations of torch in 32 bits, rounded once at the end; the recurrence by doubling:
log2(L) passes that join each token's coefficients with those of the token 2^i before it.
"""
from __future__ import annotations

import math

import torch

own = False

DEVICE = "cuda:0"
TYPES = {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}
EPS = 1e-5


# ------------------------------------------------------------------------------------------------- the cases
def _scan(op, B, L, K, N, dtype, **more):
    return dict(dict(op=op, B=B, L=L, K=K, N=N, dtype=dtype, gated=True, reverse=False, state=False, strided=False), **more)


def _conv(op, B, L, K, W, dtype, **more):
    return dict(dict(op=op, B=B, L=L, K=K, W=W, dtype=dtype, silu=True, reverse=False, state=False, strided=False), **more)


def _norm(op, B, L, K, dtype, **more):
    return dict(dict(op=op, B=B, L=L, K=K, dtype=dtype, stream="same", first=False, gate="none", post=False, scale=1.0), **more)


def listed():
    return [
        # one image through the smallest model: latency
        _scan("scan", 1, 197, 384, 16, "f16", strided=True, name="scan_ti_1_image"),
        # the largest batch of the benchmark
        _scan("scan", 256, 197, 1536, 16, "f16", name="scan_b_256_images"),
        # one long sequence, a segment of a longer one: the state comes in and goes out
        _scan("scan", 1, 16384, 768, 16, "bf16", state=True, name="scan_1_long_sequence"),
        # a training batch; the second direction of a block that reads its tokens both ways
        _scan("scan_train", 128, 197, 768, 16, "f16", reverse=True, name="scan_train_s_128_images"),
        # training on a few long documents of an odd length, all in 32 bits
        _scan("scan_train", 2, 4099, 384, 16, "f32", name="scan_train_2_long_odd"),
        # one token for each of many sequences
        _scan("scan_step", 1000, 1, 1536, 16, "bf16", name="scan_step_1000_sequences"),
        # a batch of images, the convolution's half of in_proj's output
        _conv("conv", 128, 197, 768, 4, "f16", strided=True, name="conv_s_128_images"),
        # a training batch
        _conv("conv_train", 64, 197, 1536, 4, "bf16", name="conv_train_b_64_images"),
        # one token for each of a few sequences: the smallest call
        _conv("conv_step", 16, 1, 768, 4, "f16", name="conv_step_16_sequences"),
        # the norm before each block of the largest model, the stream in 32 bits
        _norm("norm", 256, 197, 768, "f16", stream="f32", name="norm_b_256_images"),
        # training with norms on both sides and a gate for each image
        _norm("norm_train", 64, 785, 384, "bf16", gate="image", post=True, scale=0.875, name="norm_train_s_64_long_images"),
        # a few tokens of an odd width, a gate per channel
        _norm("norm", 1, 7, 1001, "f32", gate="channel", post=True, name="norm_7_tokens"),
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _width(rng, lo, hi):
    k = _log_uniform(rng, lo, hi)
    return max(lo, k // 64 * 64) if rng.random() < 0.5 else k  # half of the widths are multiples of 64


def draw(rng):
    op = rng.choice(["scan", "scan", "scan_train", "scan_train", "scan_step", "conv", "conv_train", "conv_step", "norm", "norm_train"])
    dtype = rng.choice(["f16", "f16", "bf16", "bf16", "f32"])
    reverse, state, strided = rng.random() < 0.4, rng.random() < 0.4, rng.random() < 0.4
    if op.startswith("scan"):
        N = 16 if rng.random() < 0.6 else _log_uniform(rng, 1, 64)
        most = {"scan": 5 << 27, "scan_train": 5 << 25, "scan_step": 3 << 23}[op]  # channels, states and tokens of one pass
        K = _width(rng, 16, 2048)
        L = 1 if op == "scan_step" else _log_uniform(rng, 1, min(20000, most // (K * N)))
        B = _log_uniform(rng, 1, max(1, most // (K * N * L)))
        if op == "scan_step":
            reverse = state = False
        return _scan(op, B, L, K, N, dtype, gated=rng.random() < 0.7, reverse=reverse, state=state, strided=strided)
    if op.startswith("conv"):
        most = {"conv": 3 << 24, "conv_train": 1 << 24, "conv_step": 1 << 22}[op]
        K = _width(rng, 16, 2048)
        L = 1 if op == "conv_step" else _log_uniform(rng, 1, min(20000, most // K))
        B = _log_uniform(rng, 1, max(1, most // (K * L)))
        if op == "conv_step":
            reverse = state = False
        return _conv(op, B, L, K, rng.choice([2, 3, 4, 4]), dtype, silu=rng.random() < 0.8, reverse=reverse, state=state, strided=strided)
    K = _width(rng, 16, 8192)
    most = {"norm": 5 << 23, "norm_train": 5 << 21}[op]
    L = _log_uniform(rng, 1, min(20000, most // K))
    B = _log_uniform(rng, 1, max(1, most // (K * L)))
    return _norm(op, B, L, K, dtype, stream=rng.choice(["same", "f32"]), first=rng.random() < 0.15, gate=rng.choice(["none", "channel", "image", "token"]),
                 post=rng.random() < 0.5, scale=rng.choice([1.0, 1.0, 0.875]))


# ------------------------------------------------------------------------------------------------- inputs
def _normal(g, *shape, scale=1.0):
    return torch.randn(*shape, generator=g, device=DEVICE) * scale


def _uniform(g, *shape):
    return torch.rand(*shape, generator=g, device=DEVICE)


def _half(v, width, strided):
    """`v` as the left columns of a matrix of `width` columns more, where a block's linear left it."""
    if not strided:
        return v
    wide = torch.empty((v.shape[0], v.shape[1] + width), dtype=v.dtype, device=v.device)
    wide[:, width:] = v
    return wide[:, width:]


def prepare(case, seed):
    c = dict(case)
    g = torch.Generator(device=DEVICE)
    g.manual_seed(seed)
    T = TYPES[c["dtype"]]
    B, L, K, op = c["B"], c["L"], c["K"], c["op"]
    M = B * L
    c["dy"] = _normal(g, M, K).to(T) if op.endswith("train") else None
    if op.startswith("scan"):
        N = c["N"]
        c["u"] = torch.nn.functional.silu(_normal(g, M, K)).to(T)  # what the convolution leaves
        c["dt"] = _normal(g, M, K, scale=0.5).to(T)
        step = torch.exp(_uniform(g, K) * math.log(100.0) + math.log(1e-3))  # step sizes from 0.001 to 0.1
        c["dt_bias"] = step + torch.log(-torch.expm1(-step))
        c["a"] = -torch.arange(1, N + 1, device=DEVICE, dtype=torch.float32) * torch.exp(_normal(g, K, N, scale=0.2))
        bc = _normal(g, M, 2 * N).to(T)
        bc = _half(bc, max(1, K // 32), c["strided"])  # x_proj's output: the steps' columns, then these
        c["b"], c["c"] = (bc[:, :N], bc[:, N:]) if c["strided"] else (bc[:, :N].contiguous(), bc[:, N:].contiguous())
        c["d"] = 1.0 + _normal(g, K, scale=0.1)
        c["z"] = _half(_normal(g, M, K).to(T), K, c["strided"]) if c["gated"] else None
        c["state"] = _normal(g, B, K, N, scale=0.5) if c["state"] or op == "scan_step" else None
    elif op.startswith("conv"):
        W = c["W"]
        c["x"] = _half(_normal(g, M, K).to(T), K, c["strided"])
        c["w"] = _normal(g, K, W, scale=1.0 / math.sqrt(W))
        c["bias"] = _normal(g, K, scale=0.1)
        c["state"] = _normal(g, B, W - 1, K).to(T) if c["state"] or op == "conv_step" else None
    else:
        S = T if c["stream"] == "same" else torch.float32
        c["h"] = _normal(g, M, K).to(T)
        c["residual"] = None if c["first"] else _normal(g, M, K, scale=3.0).to(S)
        groups = {"none": 0, "channel": 1, "image": B, "token": M}[c["gate"]]
        c["gate"] = 0.5 + _normal(g, groups, K, scale=0.3) if groups else None
        c["w"] = 1.0 + _normal(g, K, scale=0.1)
        c["w_post"] = 1.0 + _normal(g, K, scale=0.1) if c["post"] else None
        c["S"] = S
        if op == "norm_train":  # what the forward pass left, and the gradient from the blocks behind
            c["r"] = _norm_plain(c)[1]
            c["dr"] = _normal(g, M, K, scale=0.5).to(S)
    return c


# ------------------------------------------------------------------------------------------------- plain forms
def _softplus(p):
    return p.clamp(min=0) + torch.log1p(torch.exp(-p.abs()))


def _recur(a, x):
    """h_t = a_t h_{t-1} + x_t along dimension 1, h_{-1} = 0."""
    step = 1
    while step < a.shape[1]:
        x = torch.cat([x[:, :step], x[:, step:] + a[:, step:] * x[:, :-step]], 1)
        a = torch.cat([a[:, :step], a[:, step:] * a[:, :-step]], 1)
        step *= 2
    return x


def _tokens(v, s):
    """[B*L, X] as [B, L, X] in 32 bits and in the order of time."""
    v = v.float().view(s["B"], s["L"], -1) if v.is_contiguous() else v.float().reshape(s["B"], s["L"], -1)
    return v.flip(1) if s["reverse"] else v


def _rows(v, s):
    v = v.flip(1) if s["reverse"] else v
    return v.reshape(s["B"] * s["L"], -1).to(TYPES[s["dtype"]])


def _scan_plain(s):
    u, p = _tokens(s["u"], s), _tokens(s["dt"], s) + s["dt_bias"]
    b, c = _tokens(s["b"], s), _tokens(s["c"], s)
    D = _softplus(p)
    a = torch.exp(D[..., None] * s["a"])
    x = (D * u)[..., None] * b[:, :, None, :]
    if s["state"] is not None:
        x[:, 0] += a[:, 0] * s["state"]
    h = _recur(a, x)
    del x
    v = (h * c[:, :, None, :]).sum(-1) + s["d"] * u
    z = _tokens(s["z"], s) if s["z"] is not None else None
    y = v * z * torch.sigmoid(z) if z is not None else v
    out = {"y": _rows(y, s)}
    if s["op"] != "scan_train":
        if s["state"] is not None:
            out["state"] = h[:, -1].contiguous()
        return out

    dy = _tokens(s["dy"], s)
    if z is not None:
        sig = torch.sigmoid(z)
        out["dz"] = _rows(dy * v * sig * (1 + z * (1 - sig)), s)
        dy = dy * z * sig
    before = torch.cat([s["state"][:, None] if s["state"] is not None else torch.zeros_like(h[:, :1]), h[:, :-1]], 1)
    out["dc"] = _rows((h * dy[..., None]).sum(2), s)
    del h
    last = torch.cat([a[:, 1:], torch.zeros_like(a[:, :1])], 1)
    g = _recur(last.flip(1), (c[:, :, None, :] * dy[..., None]).flip(1)).flip(1)
    del last
    out["db"] = _rows((g * (D * u)[..., None]).sum(2), s)
    gb = (g * b[:, :, None, :]).sum(-1)
    g = g * a * before
    del a, before
    out["du"] = _rows(s["d"] * dy + D * gb, s)
    dp = (u * gb + (g * s["a"]).sum(-1)) * torch.sigmoid(p)
    out["ddt"] = _rows(dp, s)
    out["da"] = (g * D[..., None]).sum((0, 1))
    out["dd"] = (dy * u).sum((0, 1))
    out["ddt_bias"] = dp.sum((0, 1))
    return out


def _conv_plain(s):
    L, W = s["L"], s["W"]
    x = _tokens(s["x"], s)
    first = s["state"].float() if s["state"] is not None else torch.zeros_like(x[:, :1]).expand(-1, W - 1, -1)
    x = torch.cat([first, x], 1)
    p = s["bias"] + sum(x[:, j:j + L] * s["w"][:, j] for j in range(W))
    sig = torch.sigmoid(p)
    if s["op"] != "conv_train":
        out = {"y": _rows(p * sig if s["silu"] else p, s)}
        if s["state"] is not None:
            out["state"] = x[:, L:].to(TYPES[s["dtype"]])
        return out
    dp = _tokens(s["dy"], s)
    if s["silu"]:
        dp = dp * sig * (1 + p * (1 - sig))
    late = torch.cat([dp, torch.zeros_like(dp[:, :1]).expand(-1, W - 1, -1)], 1)
    return {"dx": _rows(sum(late[:, W - 1 - j:W - 1 - j + L] * s["w"][:, j] for j in range(W)), s),
            "dw": torch.stack([(dp * x[:, j:j + L]).sum((0, 1)) for j in range(W)], 1),
            "dbias": dp.sum((0, 1))}


def _gated(s):
    return None if s["gate"] is None else s["gate"].repeat_interleave(s["B"] * s["L"] // s["gate"].shape[0], 0)


def _norm_plain(s):
    q = s["h"].float()
    if s["w_post"] is not None:
        q = q * torch.rsqrt(q.square().mean(-1, keepdim=True) + EPS) * s["w_post"]
    gate = _gated(s)
    r = q if gate is None else gate * q
    if s["residual"] is not None:
        r = r + s["scale"] * s["residual"].float()
    y = r * torch.rsqrt(r.square().mean(-1, keepdim=True) + EPS) * s["w"]
    return y.to(TYPES[s["dtype"]]), r.to(s["S"])


def _norm_train_plain(s):
    def through(t, v):
        """The gradient of norm(v) . t, and norm(v)."""
        rms = torch.rsqrt(v.square().mean(-1, keepdim=True) + EPS)
        n = v * rms
        return rms * (t - n * (t * n).mean(-1, keepdim=True)), n

    T = TYPES[s["dtype"]]
    h, dy = s["h"].float(), s["dy"].float()
    dr, n = through(dy * s["w"], s["r"].float())
    dr = dr + s["dr"].float()
    out = {"dw": (dy * n).sum(0)}
    if s["residual"] is not None:
        out["dresidual"] = (s["scale"] * dr).to(s["S"])
    gate = _gated(s)
    dq = dr if gate is None else gate * dr
    q = h
    if s["w_post"] is not None:
        out["dh"], n = through(dq * s["w_post"], h)
        out["dw_post"] = (dq * n).sum(0)
        q = n * s["w_post"]
    else:
        out["dh"] = dq
    out["dh"] = out["dh"].to(T)
    if gate is not None:
        out["dgate"] = (dr * q).view(s["gate"].shape[0], -1, s["K"]).sum(1)
    return out


# ------------------------------------------------------------------------------------------------- one pass
def run(s):
    op = s["op"]
    if not own:
        if op.startswith("scan"):
            return _scan_plain(s)
        if op.startswith("conv"):
            return _conv_plain(s)
        if op == "norm_train":
            return _norm_train_plain(s)
        return dict(zip(("y", "r"), _norm_plain(s)))

    import paper_2412_20386_amd as ptq

    B, L = s["B"], s["L"]
    if op == "scan":
        after = torch.empty_like(s["state"]) if s["state"] is not None else None
        y = ptq.gated_scan(s["u"], s["dt"], s["a"], s["b"], s["c"], s["d"], s["z"], s["dt_bias"], B, L, reverse=s["reverse"], state=s["state"],
                           state_out=after)
        return {"y": y} if after is None else {"y": y, "state": after}
    if op == "scan_train":
        marks = torch.empty((ptq.scan_marks(L), B, s["K"], s["N"]), device=DEVICE)
        y = ptq.gated_scan(s["u"], s["dt"], s["a"], s["b"], s["c"], s["d"], s["z"], s["dt_bias"], B, L, reverse=s["reverse"], state=s["state"], marks=marks)
        names = ("du", "ddt", "da", "db", "dc", "dd", "dz", "ddt_bias")
        grads = ptq.gated_scan_backward(s["dy"], s["u"], s["dt"], s["a"], s["b"], s["c"], s["d"], s["z"], s["dt_bias"], marks, B, L, reverse=s["reverse"])
        return {"y": y} | {n: v for n, v in zip(names, grads) if v is not None}
    if op == "scan_step":  # the state before the token is kept, as where a drafted token may be taken back
        after = torch.empty_like(s["state"])
        y = ptq.gated_scan_step(s["u"], s["dt"], s["a"], s["b"], s["c"], s["d"], s["z"], s["dt_bias"], s["state"], state_out=after)
        return {"y": y, "state": after}
    if op == "conv":
        after = torch.empty_like(s["state"]) if s["state"] is not None else None
        y = ptq.token_conv(s["x"], s["w"], s["bias"], B, L, silu=s["silu"], reverse=s["reverse"], state=s["state"], state_out=after)
        return {"y": y} if after is None else {"y": y, "state": after}
    if op == "conv_train":
        return dict(zip(("dx", "dw", "dbias"),
                        ptq.token_conv_backward(s["dy"], s["x"], s["w"], s["bias"], B, L, silu=s["silu"], reverse=s["reverse"], state=s["state"])))
    if op == "conv_step":
        after = torch.empty_like(s["state"])
        return {"y": ptq.token_conv_step(s["x"], s["w"], s["bias"], s["state"], silu=s["silu"], state_out=after), "state": after}
    if op == "norm":
        r = torch.empty((B * L, s["K"]), dtype=s["S"], device=DEVICE)
        y, r = ptq.residual_norm(s["h"], s["residual"], s["w"], s["gate"], s["w_post"], scale=s["scale"], eps=EPS, residual_out=r)
        return {"y": y, "r": r}
    grads = ptq.residual_norm_backward(s["dy"], s["dr"], s["h"], s["r"], s["w"], s["gate"], s["w_post"], scale=s["scale"], eps=EPS,
                                       first=s["residual"] is None)
    return {n: v for n, v in zip(("dh", "dresidual", "dw", "dgate", "dw_post"), grads) if v is not None}


# ------------------------------------------------------------------------------------------------- cost
def work(case):
    """Every input once in, every output once out; for the recurrence's steps of one (token, channel, state) the product, the
    exponential, two multiply-adds and the input's product, and as many again and twice more for its gradients."""
    op, K, M = case["op"], case["K"], case["B"] * case["L"]
    e = torch.finfo(TYPES[case["dtype"]]).bits // 8
    if op.startswith("scan"):
        N, train, gated = case["N"], op == "scan_train", case["gated"]
        nbytes = M * K * e * (3 + gated) + 2 * M * N * e + 4 * K * (N + 2)
        if case["state"] or op == "scan_step":
            nbytes += 4 * case["B"] * K * N * (1 if train else 2)
        flops = M * K * (7 * N + 20)
        if train:
            nbytes += M * K * e * (3 + gated) + 2 * M * N * e + 4 * K * (N + 2)
            flops += M * K * (20 * N + 40)
        return {"bytes": nbytes, "flops": flops}
    if op.startswith("conv"):
        W, train = case["W"], op == "conv_train"
        nbytes = M * K * e * (3 if train else 2) + 4 * K * (W + 1) * (2 if train else 1)
        if case["state"] or op == "conv_step":
            nbytes += case["B"] * (W - 1) * K * e * (1 if train else 2)
        return {"bytes": nbytes, "flops": M * K * (6 * W if train else 2 * W) + M * K * (12 if train else 5)}
    r = e if case["stream"] == "same" else 4
    groups = {"none": 0, "channel": 1, "image": case["B"], "token": M}[case["gate"]]
    if op == "norm":
        return {"bytes": M * K * (2 * e + r * (1 if case["first"] else 2)) + 4 * K * (1 + case["post"] + groups), "flops": M * K * (6 + 5 * case["post"])}
    return {"bytes": M * K * (3 * e + r * (2 if case["first"] else 3)) + 8 * K * (1 + case["post"] + groups), "flops": M * K * (12 + 10 * case["post"])}


# ------------------------------------------------------------------------------------------------- in 64 bits
def exact(case, seed):
    """The definitions token by token in 64 bits; gradients by differentiating them, not by formulas."""
    s = prepare(case, seed)
    op, B, L, K = s["op"], s["B"], s["L"], s["K"]

    def time(v):  # [B, L, X] in 64 bits, tokens in the order of time
        v = v.double().reshape(B, L, -1)
        return torch.flip(v, [1]) if s.get("reverse") else v

    def back(v):
        return (torch.flip(v, [1]) if s.get("reverse") else v).reshape(B * L, -1)

    train = op.endswith("train")
    names = {"scan": ["u", "dt", "a", "b", "c", "d", "z", "dt_bias"], "conv": ["x", "w", "bias"], "norm": ["h", "residual", "w", "gate", "w_post"]}[op.split("_")[0]]
    by_token = {"u", "dt", "b", "c", "z", "x"}
    v = {n: None if s[n] is None else (time(s[n]) if n in by_token else s[n].double()).detach().requires_grad_(train) for n in names}
    with torch.set_grad_enabled(train):
        if op.startswith("scan"):
            D = torch.nn.functional.softplus(v["dt"] + v["dt_bias"], threshold=1e3)
            h = s["state"].double() if s["state"] is not None else torch.zeros((B, K, s["N"]), dtype=torch.float64, device=DEVICE)
            ys = []
            for D_t, u_t, b_t, c_t in zip(D.unbind(1), v["u"].unbind(1), v["b"].unbind(1), v["c"].unbind(1)):
                h = (D_t[:, :, None] * v["a"]).exp() * h + (D_t * u_t)[:, :, None] * b_t[:, None, :]
                ys.append(torch.matmul(h, c_t[:, :, None])[:, :, 0] if not train else (h * c_t[:, None, :]).sum(2))
            y = torch.stack(ys, 1) + v["d"] * v["u"]
            y = y if v["z"] is None else y * torch.nn.functional.silu(v["z"])
            out, loss = {"y": back(y.detach())}, (y * time(s["dy"])).sum() if train else None
            if not train and s["state"] is not None:
                out["state"] = h
        elif op.startswith("conv"):
            W = s["W"]
            first = s["state"].double() if s["state"] is not None else torch.zeros((B, W - 1, K), dtype=torch.float64, device=DEVICE)
            x = torch.cat([first, v["x"]], 1)
            y = (x.unfold(1, W, 1) * v["w"]).sum(-1) + v["bias"]
            y = torch.nn.functional.silu(y) if s["silu"] else y
            out, loss = {} if train else {"y": back(y)}, (y * time(s["dy"])).sum() if train else None
            if not train and s["state"] is not None:
                out["state"] = x[:, L:]
        else:
            unit = lambda t: t / (t.pow(2).mean(1, keepdim=True) + EPS).sqrt()  # noqa: E731
            q = v["h"] if v["w_post"] is None else unit(v["h"]) * v["w_post"]
            groups = 1 if v["gate"] is None else v["gate"].shape[0]
            r = q if v["gate"] is None else (q.view(groups, -1, K) * v["gate"][:, None, :]).reshape(-1, K)
            r = r if v["residual"] is None else r + s["scale"] * v["residual"]
            if not train:
                return {"y": unit(r) * v["w"], "r": r}
            # the stream is an input of the backward pass as the forward pass rounded it: its value, with r's gradient
            r = r + (s["r"].double() - r).detach()
            out, loss = {}, (unit(r) * v["w"] * s["dy"].double()).sum() + (r * s["dr"].double()).sum()
    if train:
        wanted = [n for n in names if v[n] is not None]
        for n, d in zip(wanted, torch.autograd.grad(loss, [v[n] for n in wanted])):
            out["d" + n] = back(d) if n in by_token else d
    return out
