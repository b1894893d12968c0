"""The recurrence on each of its layouts, by the kernels' names in the profiler's record: two channels to a lane and one, whole sequences, few chunks and
many, up to as many as there can be.  The results against bounds that have the states' own memory, so that a long sequence has no wide ones."""
import re
import warnings

import pytest
import torch
from torch.profiler import ProfilerActivity, profile

import paper_2412_20386_amd as ptq
from scan_bounds import bounds, within
from test_gpu_token_ops import BY_TOKEN, TYPES, Draw, _device, _guarded, _scan_inputs, _time

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def _ran(call):
    """(kernel, its numbers and truth values) of the recurrence's kernels that the call launched, as the profiler names them, sorted"""
    call()
    torch.cuda.synchronize()
    with warnings.catch_warnings():
        warnings.simplefilter("ignore")
        with profile(activities=[ProfilerActivity.CUDA]) as record:
            call()
            torch.cuda.synchronize()
    found = []
    for e in record.key_averages():
        name = re.search(r"gated_scan_backward_tokens|gated_scan_tokens|gated_scan_wide|gated_scan_short|join_chunks", e.key)
        if not name:
            continue
        rest = e.key[name.end():]
        if rest.startswith("<"):  # "<float, 4, 2, false, true>(..."
            # (__bf16 and a 1 behind it are read as "bool _Accum, int, E" by demanglers that do not know the type)
            values = re.findall(r"\b(\d+|true|false)\b", rest[:rest.index(">")].replace("_Accum, int, E,", "_Accum, 1,"))
        else:  # mangled: "IDF16_Li4ELi2ELb0ELb1EE..."
            values = re.findall(r"L[ib](\d+)E", rest[:rest.index("EE") + 1])
        found.append((name.group(), *(int({"true": 1, "false": 0}.get(v, v)) for v in values)))
    return sorted(found)


def _kernels(name, states, channels, ragged, chunks):
    """What a pass launches: whole, in few chunks, in many"""
    main = [(name, states, channels, ragged, 0)]
    if chunks != "whole":
        main.append((name, states, channels, ragged, 1))
    if chunks == "many":
        main.append(("join_chunks", int("backward" in name)))
    return sorted(main)


# B, L, K, N, type, reverse, state, strided, forward, backward: (states to a lane, channels to a lane, chunks)
LAYOUTS = [
    # forward with two channels to a lane: 4096 wavefronts
    (70, 18, 1900, 7, "f16", False, True, 4, (2, 2, "whole"), (2, 2, "whole")),
    (70, 18, 1900, 16, "bf16", True, True, 0, (4, 2, "whole"), (4, 2, "whole")),
    (64, 9, 2048, 16, "f16", False, False, 0, (4, 2, "whole"), (4, 2, "whole")),
    (4100, 5, 20, 4, "f32", True, True, 0, (1, 2, "whole"), (1, 2, "whole")),
    (4100, 17, 32, 8, "f16", False, True, 0, (2, 2, "whole"), (2, 2, "whole")),
    (800, 1030, 5, 3, "f16", True, True, 2, (1, 2, "few"), (1, 2, "few")),
    (26, 1030, 992, 16, "bf16", False, True, 0, (4, 2, "few"), (4, 2, "few")),
    (1, 8200, 500, 13, "f16", True, True, 1, (4, 2, "many"), (4, 2, "many")),
    (1, 16384, 768, 16, "bf16", False, True, 0, (4, 2, "many"), (4, 2, "many")),  # 256 chunks
    # backward with two channels to a lane: 2048 wavefronts
    (24, 197, 768, 16, "f16", False, True, 0, (4, 1, "whole"), (4, 2, "few")),
    (30, 200, 490, 11, "bf16", True, True, 3, (4, 1, "few"), (4, 2, "few")),
    (40, 210, 400, 5, "f32", False, False, 0, (2, 1, "few"), (2, 2, "few")),
    (2, 4099, 384, 16, "f32", False, True, 0, (4, 1, "many"), (4, 2, "many")),
    (20, 300, 500, 13, "f16", True, False, 0, (4, 1, "many"), (4, 2, "many")),
    (16, 300, 490, 4, "bf16", False, True, 0, (1, 1, "many"), (1, 2, "many")),
    # one channel to a lane
    (60, 30, 192, 16, "f16", True, True, 0, (4, 1, "whole"), (4, 1, "whole")),
    (2, 100, 40, 17, "f32", False, True, 0, (8, 1, "few"), (8, 1, "few")),
    (1, 700, 32, 32, "f16", True, True, 0, (8, 1, "many"), (8, 1, "many")),
    (1, 700, 20, 64, "bf16", False, True, 5, (16, 1, "many"), (16, 1, "many")),
    (1, 16384, 3, 2, "f32", True, True, 0, (1, 1, "many"), (1, 1, "many")),       # 256 chunks
]


@pytest.mark.parametrize("case", LAYOUTS, ids=str)
def test_layout(case):
    B, L, K, N, dtype, reverse, with_state, strided, forward, backward = case
    print("layout", case, flush=True)
    v, state = _scan_inputs(B * 1000 + L + N, B, L, K, N, dtype, state=with_state)
    T, M = TYPES[dtype], B * L
    gpu = {k: _device(t, strided if k in BY_TOKEN else 0) for k, t in v.items()}
    y, untouched = _guarded(M, K, T)
    state_out, marks, first = torch.empty((B, K, N), device=DEV), torch.empty((ptq.scan_marks(L), B, K, N), device=DEV), _device(state)
    ragged = lambda channels, states: int(K % (16 * channels) != 0 or N != 4 * states)  # noqa: E731
    ran = _ran(lambda: ptq.gated_scan(*gpu.values(), B, L, reverse=reverse, state=first, y=y, state_out=state_out, marks=marks))
    assert ran == _kernels("gated_scan_tokens", forward[0], forward[1], ragged(forward[1], forward[0]), forward[2])
    untouched()
    dy = _device(Draw(7)(M, K, dtype=T), strided)
    grads = []
    ran = _ran(lambda: grads.append(ptq.gated_scan_backward(dy, *gpu.values(), marks, B, L, reverse=reverse)))
    assert ran == _kernels("gated_scan_backward_tokens", backward[0], backward[1], ragged(backward[1], backward[0]), backward[2])

    exact = {k: _time(t, B, L, reverse) if k in BY_TOKEN else t.double() for k, t in gpu.items()}
    want = bounds(_time(dy, B, L, reverse), **exact, state=None if first is None else first.double(), chunk=max(160, L if "whole" in (forward[2], backward[2]) else 0))
    got = dict(zip(("du", "ddt", "da", "db", "dc", "dd", "dz", "ddt_bias"), grads[0]), y=y, state_out=state_out, marks=marks)
    parts = {}
    for k, t in got.items():
        by_token = k in ("y", "du", "ddt", "db", "dc", "dz")
        parts[k] = within(_time(t, B, L, reverse) if by_token else t.double(), *want[k], T if by_token else torch.float32)
    print({k: round(p, 3) for k, p in parts.items()}, flush=True)
    assert all(p <= 1 for p in parts.values()), parts
    assert all(torch.equal(a, b) for a, b in zip(*grads))  # the same inputs: the same bits
