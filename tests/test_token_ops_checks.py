"""What the operators between a block's linears refuse before any launch: at the C boundary (pointers that are never read) and in
the Python callables (fake CUDA tensors without storage)."""
import os

import pytest
import torch
from torch._subclasses.fake_tensor import FakeTensorMode

import paper_2412_20386_amd as ptq
from paper_2412_20386_amd import build as hip_build

# A check that went missing would launch a kernel on these addresses: only where there is nothing to launch on
pytestmark = pytest.mark.skipif(torch.cuda.is_available(), reason="runs without a GPU")

P, ODD = 0x10000, 0x10001  # never dereferenced: every check below fails before a launch
NULL, SHAPE, STRIDE, ALIGN = -1, -2, -3, -4
HUGE = 1 << 50


@pytest.fixture(scope="module")
def lib():
    if not (os.path.exists(ptq.binding.LIB_PATH) and os.path.exists(ptq.binding.CALLS_PATH)):
        hip_build.build()
    return ptq.binding.load()


B, L, K, N, W = 2, 5, 48, 16, 4
SIZES = dict(B=B, L=L, K=K, N=N)
# every entry point's arguments in order, a valid call (but for the addresses); pointers: P
CALLS = {
    "gated_scan": dict(dtype=0, u=P, dt=P, a=P, b=P, c=P, d=P, z=P, dt_bias=P, state=P, y=P, state_out=P, marks=P, workspace=P, workspace_bytes=HUGE, reverse=0, **SIZES,
                       ldu=K, lddt=K, ldb=N, ldc=N, ldz=K, ldy=K, stream=None),
    "gated_scan_backward": dict(dtype=0, dy=P, u=P, dt=P, a=P, b=P, c=P, d=P, z=P, dt_bias=P, marks=P, du=P, ddt=P, da=P, db=P, dc=P, dd=P, dz=P, ddt_bias=P, workspace=P,
                                workspace_bytes=HUGE, reverse=0, **SIZES, lddy=K, ldu=K, lddt=K, ldb=N, ldc=N, ldz=K, lddu=K, ldddt=K, lddb=N, lddc=N, lddz=K, stream=None),
    "gated_scan_step": dict(dtype=0, u=P, dt=P, a=P, b=P, c=P, d=P, z=P, dt_bias=P, state=P, y=P, state_out=P, B=B, K=K, N=N, ldu=K, lddt=K, ldb=N, ldc=N, ldz=K, ldy=K,
                            stream=None),
    "token_conv": dict(dtype=0, x=P, w=P, bias=P, state=P, y=P, state_out=P, silu=1, reverse=0, B=B, L=L, K=K, W=W, ldx=K, ldy=K, stream=None),
    "token_conv_backward": dict(dtype=0, dy=P, x=P, w=P, bias=P, state=P, dx=P, dw=P, dbias=P, workspace=P, workspace_bytes=HUGE, silu=1, reverse=0, B=B, L=L, K=K, W=W,
                                lddy=K, ldx=K, lddx=K, stream=None),
    "token_conv_step": dict(dtype=0, x=P, w=P, bias=P, state=P, y=P, state_out=P, silu=1, B=B, K=K, W=W, ldx=K, ldy=K, stream=None),
    "residual_norm": dict(dtype=0, stream_dtype=0, h=P, residual=P, w=P, gate=P, w_post=P, y=P, r=P, scale=1.0, eps=1e-5, M=10, K=K, G=2, ldh=K, ldres=K, ldy=K, ldr=K,
                          stream=None),
    "residual_norm_backward": dict(dtype=0, stream_dtype=0, dy=P, dr=P, h=P, r=P, w=P, gate=P, w_post=P, dh=P, dresidual=P, dw=P, dgate=P, dw_post=P, workspace=P,
                                   workspace_bytes=HUGE, scale=1.0, eps=1e-5, M=10, K=K, G=2, lddy=K, lddr=K, ldh=K, ldr=K, lddh=K, lddres=K, stream=None),
}
OPTIONAL = {"gated_scan": "d z dt_bias state state_out marks workspace", "gated_scan_backward": "d z dt_bias dd dz ddt_bias", "gated_scan_step": "d z dt_bias",
            "token_conv": "bias state state_out", "token_conv_backward": "bias state dbias", "token_conv_step": "bias",
            "residual_norm": "residual gate w_post", "residual_norm_backward": "dr gate w_post dresidual dgate dw_post"}


def call(lib, name, **changed):
    return getattr(lib, "ptq4vm_" + name)(*(CALLS[name] | changed).values())


def pointers(name):
    return [k for k, v in CALLS[name].items() if v == P]


@pytest.mark.parametrize("name", CALLS)
def test_pointers(lib, name):
    assert len(CALLS[name]) == len(getattr(lib, "ptq4vm_" + name).argtypes)
    for k in pointers(name):
        if k not in OPTIONAL[name].split():
            assert call(lib, name, **{k: None}) == NULL, k
        assert call(lib, name, **{k: ODD}) == ALIGN, k
    for given, gradient in (("d", "dd"), ("z", "dz"), ("dt_bias", "ddt_bias"), ("gate", "dgate"), ("w_post", "dw_post")):
        if gradient in CALLS[name]:
            assert call(lib, name, **{gradient: None}) == NULL, gradient


@pytest.mark.parametrize("name", CALLS)
def test_sizes(lib, name):
    sizes = {k: v for k, v in CALLS[name].items() if k in ("B", "L", "K", "N", "W", "M")}
    for k in sizes:
        assert call(lib, name, **{k: -1}) == SHAPE, k
        assert call(lib, name, **{k: 1 << 40}) == SHAPE, k
        if k not in ("B", "M"):
            assert call(lib, name, **{k: 0}) == SHAPE, k
    for dtype in (-1, 3):
        assert call(lib, name, dtype=dtype) == SHAPE
    if "N" in sizes:
        assert call(lib, name, N=65) == SHAPE
    if "W" in sizes:
        assert call(lib, name, W=1) == SHAPE and call(lib, name, W=5) == SHAPE
    if "G" in CALLS[name]:
        assert call(lib, name, G=3) == SHAPE and call(lib, name, G=0) == SHAPE and call(lib, name, G=-2) == SHAPE
        assert call(lib, name, K=16385) == SHAPE
        assert call(lib, name, dtype=0, stream_dtype=1) == SHAPE and call(lib, name, dtype=2, stream_dtype=0) == SHAPE
    if name == "gated_scan_step":
        assert call(lib, name, B=1 << 24, K=1, ldu=1, lddt=1, ldz=1, ldy=1) == SHAPE  # more threads than a grid holds
    # B * L beyond 31 bits, each of them below
    if "L" in sizes:
        assert call(lib, name, B=1 << 20, L=1 << 20) == SHAPE


@pytest.mark.parametrize("name", CALLS)
def test_pitches(lib, name):
    for k, v in CALLS[name].items():
        if k.startswith("ld"):
            assert call(lib, name, **{k: v - 1}) == STRIDE, k
            assert call(lib, name, **{k: -v}) == STRIDE, k
            if name.startswith("gated_scan"):
                assert call(lib, name, **{k: 1 << 26}) == STRIDE, k  # offsets inside a few tokens are 32-bit


def test_workspaces(lib):
    need = {"gated_scan_backward": lib.ptq4vm_gated_scan_backward_workspace(B, L, K, N), "token_conv_backward": lib.ptq4vm_token_conv_backward_workspace(B, L, K, W),
            "residual_norm_backward": lib.ptq4vm_residual_norm_backward_workspace(10, K, 2)}
    for name, n in need.items():
        assert 0 < n < 1 << 20 and call(lib, name, workspace_bytes=n - 1) == SHAPE, name
    assert lib.ptq4vm_gated_scan_workspace(B, L, K, N) == 0  # one chunk
    n = lib.ptq4vm_gated_scan_workspace(1, 5000, K, N)
    assert n > 0
    assert call(lib, "gated_scan", B=1, L=5000, workspace=None, workspace_bytes=0) == NULL
    assert call(lib, "gated_scan", B=1, L=5000, workspace_bytes=n - 1) == SHAPE
    # sizes that the entry points refuse need none
    assert lib.ptq4vm_gated_scan_workspace(-1, L, K, N) == 0 and lib.ptq4vm_gated_scan_backward_workspace(B, L, K, 65) == 0
    assert lib.ptq4vm_token_conv_backward_workspace(B, 0, K, W) == 0 and lib.ptq4vm_residual_norm_backward_workspace(10, K, 3) == 0


def test_nothing_to_do(lib):
    for name in ("gated_scan", "gated_scan_step", "token_conv", "token_conv_step"):
        assert call(lib, name, B=0) == 0
    assert call(lib, "gated_scan", B=0, u=None, dt=None, b=None, c=None, y=None) == 0  # matrices of no rows
    assert call(lib, "residual_norm", M=0) == 0


# ---------------------------------------------------------------------------------- the Python callables
F, H, BF, D64 = torch.float32, torch.float16, torch.bfloat16, torch.float64


def fake(dtype, *shape, device="cuda:0"):
    with FakeTensorMode(allow_non_fake_inputs=True):
        return torch.empty(shape, dtype=dtype, device=device)


M = B * L
m = lambda *s, t=H: fake(t, *s)  # noqa: E731
f = lambda *s: fake(F, *s)  # noqa: E731
SCAN = dict(u=m(M, K), dt=m(M, K), a=f(K, N), b=m(M, N), c=m(M, N), d=f(K), z=m(M, K), dt_bias=f(K))
PYTHON = {
    "gated_scan": (SCAN | dict(B=B, L=L), dict(state=f(B, K, N), y=m(M, K), state_out=f(B, K, N), marks=f(1, B, K, N))),
    "gated_scan_backward": (dict(dy=m(M, K)) | SCAN | dict(marks=f(1, B, K, N), B=B, L=L), dict(du=m(M, K), ddt=m(M, K), db=m(M, N), dc=m(M, N), dz=m(M, K))),
    "gated_scan_step": ({k: (m(B, v.shape[1]) if v.dtype == H else v) for k, v in SCAN.items()} | dict(state=f(B, K, N)), dict(y=m(B, K), state_out=f(B, K, N))),
    "token_conv": (dict(x=m(M, K), w=f(K, W), bias=f(K), B=B, L=L), dict(state=m(B, W - 1, K), y=m(M, K), state_out=m(B, W - 1, K))),
    "token_conv_backward": (dict(dy=m(M, K), x=m(M, K), w=f(K, W), bias=f(K), B=B, L=L), dict(state=m(B, W - 1, K), dx=m(M, K))),
    "token_conv_step": (dict(x=m(B, K), w=f(K, W), bias=f(K), state=m(B, W - 1, K)), dict(y=m(B, K), state_out=m(B, W - 1, K))),
    "residual_norm": (dict(h=m(M, K), residual=f(M, K), w=f(K)), dict(gate=f(2, K), w_post=f(K), y=m(M, K), residual_out=f(M, K))),
    "residual_norm_backward": (dict(dy=m(M, K), dr=f(M, K), h=m(M, K), r=f(M, K), w=f(K)), dict(gate=f(2, K), w_post=f(K), dh=m(M, K), dresidual=f(M, K))),
}


@pytest.mark.parametrize("name", PYTHON)
def test_valid_calls_get_as_far_as_the_launch(lib, name):
    required, optional = PYTHON[name]
    for kw in (required, required | optional):
        with pytest.raises(RuntimeError) as err:  # no device here, no storage anywhere
            getattr(ptq, name)(**kw)
        assert not isinstance(err.value, ptq.Ptq4vmError)


@pytest.mark.parametrize("name", PYTHON)
def test_tensors_of_other_types_and_shapes_are_refused(lib, name):
    required, optional = PYTHON[name]
    whole = required | optional
    fn = getattr(ptq, name)
    for k, t in whole.items():
        if not isinstance(t, torch.Tensor):
            continue
        shape = tuple(t.shape)
        bad = [fake(D64, *shape), fake(t.dtype, *shape, device="cpu"), fake(t.dtype, *shape, 1), fake(t.dtype, *shape[::-1]).permute(*reversed(range(t.dim())))]
        if t.dim() == 1:
            bad.pop()  # a vector is its own transpose
        bad += [fake(t.dtype, *shape[:i], n - 1, *shape[i + 1:]) for i, n in enumerate(shape) if n > 1 and (k, i) != ("gate", 0)]  # (one gate would do)
        if t.dtype == H:
            bad.append(fake(BF, *shape))
        bad.append("a tensor")
        bad.append(fake(t.dtype, *shape, device="cuda:1"))  # not where the others are
        for wrong in bad:
            with pytest.raises((TypeError, ValueError)):
                fn(**(whole | {k: wrong}))


@pytest.mark.parametrize("name", PYTHON)
def test_arguments(lib, name):
    required, optional = PYTHON[name]
    fn = getattr(ptq, name)
    with pytest.raises(TypeError, match="unexpected keyword argument 'nothing'"):
        fn(**required, nothing=1)
    with pytest.raises(TypeError, match="missing required argument"):
        fn(*list(required.values())[:-1])
    if "B" in required:
        for b, l in ((B + 1, L), (1 << 62, 4), (-B, -L), (B * L, 0)):
            with pytest.raises(ValueError):
                fn(**(required | dict(B=b, L=l)))
        with pytest.raises(TypeError):
            fn(**(required | dict(B=2.5)))


def test_what_belongs_together(lib):
    required, _ = PYTHON["gated_scan_backward"]
    with pytest.raises(ValueError, match="dz"):
        ptq.gated_scan_backward(**(required | dict(z=None)), dz=m(M, K))
    required, optional = PYTHON["residual_norm_backward"]
    with pytest.raises(ValueError, match="dresidual"):
        ptq.residual_norm_backward(**required, first=True, dresidual=f(M, K))
    required, _ = PYTHON["residual_norm"]
    with pytest.raises(ValueError, match="gate"):
        ptq.residual_norm(**required, gate=f(3, K))
