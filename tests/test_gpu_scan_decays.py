"""The recurrence where a decay leaves the range of fp32, on every layout and way of joining chunks."""
import pytest
import torch

import paper_2412_20386_amd as ptq
from scan_bounds import bounds, within
from test_gpu_token_ops import BY_TOKEN, TYPES, Draw, _device, _scan_inputs, _time

pytestmark = pytest.mark.gpu
DEV = "cuda:0"

# B, L, K, N, type, reverse: lengths that end inside a tile and inside a group of tokens; fewer chunks than a run joins
SIZES = [
    (2, 15, 33, 16, "f16", False),     # whole, one tile
    (1, 1, 16, 16, "f32", False),
    (1, 65, 16, 33, "bf16", True),     # few chunks
    (1, 600, 18, 16, "f32", False),    # many chunks
    (1, 333, 40, 64, "f16", True),
    (1, 197, 48, 16, "f16", False),    # the tiles of a sequence side by side
    (3, 43, 17, 5, "f32", True),
    (4100, 3, 64, 16, "bf16", False),  # a channel to a lane
    (4100, 13, 20, 11, "f32", True),
    (4100, 5, 40, 8, "f16", False),    # two channels to a lane
    (40, 210, 400, 5, "f32", False),
]


def _check(v, state, dy, B, L, reverse, T, chunk=160, reference=lambda a: a):
    gpu = {k: _device(t) for k, t in v.items()}
    first = _device(state)
    K, N = gpu["a"].shape
    state_out, marks = torch.empty((B, K, N), device=DEV), torch.empty((ptq.scan_marks(L), B, K, N), device=DEV)
    y = ptq.gated_scan(*gpu.values(), B, L, reverse=reverse, state=first, state_out=state_out, marks=marks)
    grads = ptq.gated_scan_backward(_device(dy), *gpu.values(), marks, B, L, reverse=reverse)
    exact = {k: None if t is None else _time(t, B, L, reverse) if k in BY_TOKEN else t.double() for k, t in gpu.items()}
    exact["a"] = reference(exact["a"])
    want = bounds(_time(_device(dy), B, L, reverse), **exact, state=None if first is None else first.double(), chunk=chunk)
    got = dict(zip(("du", "ddt", "da", "db", "dc", "dd", "dz", "ddt_bias"), grads), y=y, state_out=state_out, marks=marks)
    parts = {}
    for k, t in got.items():
        if want[k] is None:
            assert t is None, k
            continue
        by_token = k in ("y", "du", "ddt", "db", "dc", "dz")
        value, error = want[k]
        parts[k] = within(_time(t, B, L, reverse) if by_token else t.double(), value, error, T if by_token else torch.float32)
    print({k: round(p, 3) for k, p in parts.items()}, flush=True)
    assert all(p <= 1 for p in parts.values()), parts


def _forgetting(a):
    """Some states that keep nothing: rates of minus infinity, and finite ones that log2(e) times are beyond fp32"""
    a = a.clone()
    a[:, 0] = float("-inf")
    a.view(-1)[1::3] = -3.3e38
    a.view(-1)[2::5] = -2.4e38
    return a


@pytest.mark.parametrize("case", SIZES, ids=str)
def test_states_that_keep_nothing(case):
    """e^{D a} is 0 for every token that there is: what is staged behind the last token, or joined behind the last chunk, leaves them alone."""
    B, L, K, N, dtype, reverse = case
    print("decays", case, flush=True)
    v, state = _scan_inputs(L, B, L, K, N, dtype, state=True)
    v["a"] = _forgetting(v["a"])
    # (0 times infinity has no value; a rate of -1e300 makes the same decay)
    _check(v, state, Draw(3)(B * L, K, dtype=TYPES[dtype]), B, L, reverse, TYPES[dtype], chunk=max(160, L), reference=lambda a: a.clamp(min=-1e300))


@pytest.mark.parametrize("B,K,N,dtype", [(3, 50, 16, "f16"), (2, 33, 5, "f32"), (5, 20, 64, "bf16"), (2, 30, 8, "f32"), (2, 9, 37, "f16")])
def test_states_that_keep_nothing_step_by_step(B, K, N, dtype):
    v, state = _scan_inputs(11, B, 1, K, N, dtype, state=True)
    v["a"] = _forgetting(v["a"])
    gpu, now = {k: t.to(DEV) for k, t in v.items()}, state.to(DEV)
    y = ptq.gated_scan_step(*gpu.values(), now)
    exact = {k: _time(t, B, 1, False) if k in BY_TOKEN else t.double() for k, t in gpu.items()}
    exact["a"] = exact["a"].clamp(min=-1e300)
    want = bounds(torch.zeros_like(exact["u"]), **exact, state=state.to(DEV).double())
    assert within(_time(y, B, 1, False), *want["y"], TYPES[dtype]) <= 1 and within(now, *want["state_out"], torch.float32) <= 1


@pytest.mark.parametrize("with_state", [False, True])
@pytest.mark.parametrize("L,N,reverse", [(100, 17, False), (600, 16, True), (200, 16, False), (200, 3, True), (333, 64, False)])
def test_states_that_grow_over_a_chunk(L, N, reverse, with_state):
    """A state grows by e^100, beyond the range of fp32, over 16 tokens, where it and the gradients are small or zero: its values are finite, and so
    are those of sequences in chunks, whose decays over a chunk are one number."""
    B, K = 1, 20
    print("growth", L, N, reverse, with_state, flush=True)
    v, _ = _scan_inputs(L + N, B, L, K, N, "f32", bias=False)
    v["dt"] = v["dt"] * 0.5 - 7  # steps of about 0.001
    v["dt"][32:48], v["u"][:64] = 100 / 16, 0.0  # (softplus(6.25) = 6.252)
    v["a"][:, N // 2] = 1.0
    state = torch.full((B, K, N), 1e-35) if with_state else None
    dy = Draw(5)(L, K) * 1e-30
    if reverse:  # the same in the order of time
        for k in BY_TOKEN:
            v[k] = v[k].flip(0).contiguous()
        dy = dy.flip(0).contiguous()
    _check(v, state, dy, B, L, reverse, torch.float32)
