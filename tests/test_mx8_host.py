"""What the 8-bit operators refuse, and the helpers of their tests (CPU)."""
import ctypes
import os

import pytest
import torch

from paper_2607_05711_amd import _lib
from tests import _mx8 as ref

built = pytest.mark.skipif(not os.path.exists(_lib.LIB_PATH) or torch.cuda.is_available(),
                           reason="host-logic checks with fake pointers run without a GPU, on the built library")
A, B, ODD, N0 = ctypes.c_void_p(0x100000), ctypes.c_void_p(0x200000), ctypes.c_void_p(0x100008), None   # never dereferenced


@built
def test_norm_refusals():
    def f(x=A, res=N0, w=A, rows=4, cols=64, eps=1e-6, h=N0, y=N0, codes=A, scales=A, rstd=N0):
        return _lib.load().ft_rmsnorm_quantize8(x, res, w, rows, cols, eps, h, y, codes, scales, rstd, N0)
    assert f(cols=48) == f(rows=-1) == f(rows=(1 << 30) + 1) == _lib.FT_ERR_SHAPE
    assert f(cols=16416) == f(eps=-1.0) == f(eps=float("nan")) == _lib.FT_ERR_UNSUPPORTED
    assert f(res=A) == f(h=A) == _lib.FT_ERR_UNSUPPORTED            # h with a residual, and only then
    assert f(x=N0) == f(w=N0) == f(scales=N0) == f(codes=N0) == f(codes=N0, scales=N0) == _lib.FT_ERR_NULL
    for k in ("x", "w", "y", "codes", "scales", "rstd"):
        assert f(**{k: ODD}) == _lib.FT_ERR_ALIGN, k
    assert f(res=ODD, h=A) == f(res=A, h=ODD) == _lib.FT_ERR_ALIGN
    assert f(rows=0) == f(cols=0) == _lib.FT_OK


@built
def test_norm_bwd_refusals():
    L = _lib.load()
    def f(dy=A, dh=N0, h=A, w=A, rstd=A, rows=4, cols=64, dx=A, dw=N0, ws=N0, n=0):  # noqa: E306
        return L.ft_rmsnorm_bwd(dy, dh, h, w, rstd, rows, cols, dx, dw, ws, n, N0)
    assert f(cols=48) == f(rows=-1) == _lib.FT_ERR_SHAPE
    assert f(cols=16416) == _lib.FT_ERR_UNSUPPORTED
    for k in ("dy", "h", "w", "rstd", "dx"):
        assert f(**{k: N0}) == _lib.FT_ERR_NULL and f(**{k: ODD}) == _lib.FT_ERR_ALIGN, k
    need = L.ft_rmsnorm_bwd_workspace_size(4, 64)
    assert need >= 64 * 4 and L.ft_rmsnorm_bwd_workspace_size(0, 64) == 0
    assert f(dw=A) == _lib.FT_ERR_NULL and f(dw=A, ws=B, n=need - 1) == _lib.FT_ERR_SHAPE
    assert f(dw=A, ws=ODD, n=need) == f(dw=ODD, ws=B, n=need) == f(dh=ODD) == _lib.FT_ERR_ALIGN
    assert f(rows=0) == f(cols=0) == _lib.FT_OK


@built
def test_quantize_refusals():
    L = _lib.load()
    def f(src=A, z=N0, act=0, rows=4, cols=64, v=N0, codes=A, scales=A, proj=N0, R=0, layout=0, out=N0, ws=N0, n=0):  # noqa: E306
        return L.ft_quantize8(src, z, act, rows, cols, v, codes, scales, proj, R, layout, out, ws, n, N0)
    assert f(cols=48) == f(rows=-1) == _lib.FT_ERR_SHAPE
    assert f(cols=(1 << 20) + 32) == f(act=4, z=A) == f(act=1) == f(z=A) == f(v=A) == _lib.FT_ERR_UNSUPPORTED
    assert f(z=A, act=1, proj=A, R=16, out=A) == f(proj=A, R=20, out=A) == f(proj=A, R=144, out=A) == _lib.FT_ERR_UNSUPPORTED
    assert f(layout=2) == f(proj=A, R=16, out=A, layout=7) == f(proj=A) == _lib.FT_ERR_UNSUPPORTED
    assert f(src=N0) == f(codes=N0) == f(scales=N0) == f(proj=A, R=16) == _lib.FT_ERR_NULL
    assert f(src=ODD) == f(codes=ODD) == f(scales=ODD) == f(z=ODD, act=2) == f(z=A, act=2, v=ODD) == _lib.FT_ERR_ALIGN
    assert f(proj=ODD, R=16, out=A) == f(proj=A, R=16, out=ODD) == _lib.FT_ERR_ALIGN
    need = L.ft_quantize8_workspace_size(4, 4096, 16, 0)
    if need:
        assert f(cols=4096, proj=A, R=16, out=A) == _lib.FT_ERR_NULL
        assert f(cols=4096, proj=A, R=16, out=A, ws=B, n=need - 1) == _lib.FT_ERR_SHAPE
    assert f(rows=0) == f(cols=0) == _lib.FT_OK


@built
@pytest.mark.parametrize("back", [False, True])
def test_linear_refusals(back):
    L = _lib.load()

    def f(x=A, xs=A, M=4, N=64, K=96, wq=A, ws=A, P=N0, R=0, F=N0, act=0, res=N0, z=N0, out=A, dt=0, bias=N0):
        if back:
            return L.ft_linear8_bwd_input(x, xs, M, N, wq, ws, K, P, R, F, z, act, res, out, dt, N0)
        return L.ft_linear8_fwd(x, xs, M, K, wq, ws, N, P, R, F, bias, act, res, z, out, dt, N0)
    assert f(M=-1) == f(N=48) == f(K=48) == f(**{"N" if back else "K": 0}) == _lib.FT_ERR_SHAPE
    assert f(dt=2) == f(act=4) == f(act=-1) == _lib.FT_ERR_UNSUPPORTED
    assert f(P=A, F=A, R=20) == f(P=A, F=A, R=144) == f(P=A, F=A) == _lib.FT_ERR_UNSUPPORTED
    if back:
        assert f(act=1) == f(z=A) == _lib.FT_ERR_UNSUPPORTED
    for k in ("x", "xs", "wq", "ws", "out"):
        assert f(**{k: N0}) == _lib.FT_ERR_NULL and f(**{k: ODD}) == _lib.FT_ERR_ALIGN, k
    assert f(res=ODD) == f(z=ODD, act=1) == f(P=ODD, F=A, R=16) == f(P=A, F=ODD, R=16) == _lib.FT_ERR_ALIGN
    assert f(P=A, R=16) == f(F=A, R=16) == _lib.FT_ERR_NULL
    i = "N" if back else "K"
    assert f(**{i: 65536 + 32}) == f(**{"K" if back else "N": (1 << 20) + 32}) == _lib.FT_ERR_UNSUPPORTED
    assert f(N=65536, K=65536) == _lib.FT_ERR_UNSUPPORTED               # N K / 2 = 2 GiB
    assert f(M=1 << 25, **{i: 2048}) == _lib.FT_ERR_UNSUPPORTED         # 2 GiB of scales
    assert f(M=(1 << 22) + 1, **{i: 32, "K" if back else "N": 1 << 20}) == _lib.FT_ERR_UNSUPPORTED
    assert f(M=0) == f(**{"K" if back else "N": 0}) == _lib.FT_OK


def test_bindings_check_their_tensors():
    """Types, shapes and devices are refused before anything is loaded or launched on them."""
    x = torch.zeros((4, 64), dtype=torch.bfloat16)
    q, s = torch.zeros((4, 64), dtype=torch.float8_e4m3fn), torch.zeros((1, 4, 4), dtype=torch.uint8)
    w = torch.zeros((32, 32), dtype=torch.uint8)
    if not os.path.exists(_lib.LIB_PATH):
        pytest.skip("libfourtune.so not built")
    for call in (lambda: _lib.ft_rmsnorm_quantize8(x.float(), x[0]), lambda: _lib.ft_quantize8(x.half()),
                 lambda: _lib.ft_linear8_fwd(q.view(torch.uint8), s, w, s), lambda: _lib.ft_rmsnorm_bwd(x.float(), x, x[0], x[0])):
        with pytest.raises(TypeError):
            call()
    for call in (lambda: _lib.ft_rmsnorm_quantize8(x, x[0]), lambda: _lib.ft_quantize8(x),
                 lambda: _lib.ft_linear8_fwd(q, s, w, s), lambda: _lib.ft_linear8_bwd_input(q, s, w, s)):
        with pytest.raises(ValueError, match="GPU"):
            call()


# ------------------------------------------------------------- the references
def test_reference_block_rule():
    """Nearest search on the table agrees with torch's E4M3 rounding; the scale is the smallest that does not clip."""
    g = torch.Generator().manual_seed(1)
    x = torch.randn((64, 256), generator=g).to(torch.bfloat16)
    c, s = ref.mxfp8(x)
    e = s.transpose(0, 1).reshape(64, -1).int() - 127
    t = (x.double().unflatten(1, (-1, 32)) / ref.pow2(e)[..., None])
    assert float(t.abs().max()) <= 448 and bool((t.abs().amax(2) > 224).all())
    assert torch.equal(t.float().to(torch.float8_e4m3fn).view(torch.uint8).flatten(1), c)
    assert torch.equal(ref.values8(c.view(torch.float8_e4m3fn), s), (c.view(torch.float8_e4m3fn).double().unflatten(1, (-1, 32)) * ref.pow2(e)[..., None]).flatten(1))
    v = ref.e4m3_values()
    assert v[-1] == 448 and v[1] == 2.0 ** -9 and bool((v[1:] > v[:-1]).all())
    assert torch.equal(torch.arange(127, dtype=torch.uint8).view(torch.float8_e4m3fn).double(), v)


@pytest.mark.parametrize("act", [1, 2, 3])
def test_reference_activation_gradients(act):
    z = torch.linspace(-6, 6, 241, dtype=torch.float64) + 0.013
    h = 1e-5
    diff = (ref.act64(act, z + h) - ref.act64(act, z - h)) / (2 * h)
    assert float((diff - ref.act_grad64(act, z)).abs().max()) < 1e-8


def test_reference_norm_gradients_against_differences():
    g = torch.Generator().manual_seed(2)
    h, dy, dh = (torch.randn((3, 64), generator=g, dtype=torch.float64) for _ in range(3))
    w, eps = torch.randn(64, generator=g, dtype=torch.float64), 1e-3

    def f(h, w):
        return float((h * torch.rsqrt(h.square().mean(1, keepdim=True) + eps) * w * dy).sum() + (h * dh).sum())
    rstd = torch.rsqrt(h.square().mean(1) + eps)
    dx, dw = ref.norm_bwd64(dy, h, w, rstd, dh)
    for t, d in ((h, dx), (w, dw)):
        for _ in range(20):
            u = torch.randn(t.shape, generator=g, dtype=torch.float64)
            plus, minus = ((t + s * 1e-5 * u) for s in (1, -1))
            diff = (f(plus, w) - f(minus, w)) / 2e-5 if t is h else (f(h, plus) - f(h, minus)) / 2e-5
            assert abs(diff - float((d * u).sum())) < 1e-6 * (1 + abs(diff))


def test_no_rows_with_an_activation():
    """Empty tensors have no address: no rows is a no-op whatever goes with them."""
    L = _lib.load()
    assert L.ft_quantize8(None, None, _lib.FT_ACT_GELU, 0, 64, None, None, None, None, 0, 0, None, None, 0, None) == _lib.FT_OK
    assert L.ft_linear8_bwd_input(None, None, 0, 64, None, None, 32, None, 0, None, None, _lib.FT_ACT_SILU, None, None,
                                  _lib.FT_BF16, None) == _lib.FT_OK


@built
@pytest.mark.parametrize("back", [False, True])
def test_more_outputs_than_a_launch_holds(back):
    """2^39 outputs, four times what the card's memory holds: past 2^24 workgroups a launch would run some of them only."""
    L = _lib.load()
    for M, o in ((1 << 20, 1 << 20), (1 << 19, 1 << 20), (1 << 28, 1 << 11)):
        if back:
            s = L.ft_linear8_bwd_input(A, A, M, 32, A, A, o, N0, 0, N0, N0, 0, N0, A, 0, N0)
        else:
            s = L.ft_linear8_fwd(A, A, M, 32, A, A, o, N0, 0, N0, N0, 0, N0, N0, A, 0, N0)
        assert s == _lib.FT_ERR_UNSUPPORTED


@built
def test_rows_kernel_has_no_instance_that_no_call_reaches():
    """More than 16 rows go there with at most 8192 columns, where a workgroup takes 16 or 32 of them."""
    names = open(_lib.LIB_PATH, "rb").read()
    assert all(b"k_rows_mx8ILi%dELi%dE" % mn in names for mn in ((1, 1), (1, 2), (1, 4), (2, 1), (2, 2)))
    assert b"k_rows_mx8ILi2ELi4E" not in names


@built
@pytest.mark.parametrize("back,M,K,N,want", [
    # few rows: the forward's kernel for them (1), up to 16 rows, and up to 32 of at most 8192 columns
    (False, 1, 4096, 4096, 1), (False, 16, 4096, 16384, 1), (False, 17, 4096, 8192, 1), (False, 32, 4096, 8192, 1),
    (False, 17, 4096, 8224, 64), (False, 32, 4096, 16384, 64), (False, 33, 4096, 4096, 64), (True, 1, 4096, 4096, 64),
    # the sizes whose times on all four tiles stand at the rule
    (False, 4608, 4096, 16384, 192), (False, 4608, 16384, 4096, 192), (False, 18432, 4096, 16384, 256),
    (False, 2048, 4096, 4096, 128), (False, 512, 4096, 4096, 64), (True, 4608, 4096, 16384, 192),
    # 416 stages are the most whose weight scales fit beside the ring of a 256x256 tile; past them two rounds of
    # 128x128 tiles (4 + 0.83 us a stage) come before two of 192x256 (7 + 0.93)
    (False, 16384, 53248, 1024, 256), (False, 16384, 53280, 1024, 128), (True, 16384, 1024, 53248, 256),
    (True, 16384, 1024, 53280, 128),
])
def test_kernel_of_a_product(back, M, K, N, want):
    f = _lib.load().ftx_linear8_tile
    f.argtypes, f.restype = [ctypes.c_int] + [ctypes.c_int64] * 3, ctypes.c_int
    assert f(int(back), M, N, K) == want


def test_workspaces_that_a_kernel_cannot_write():
    """A workspace in host memory, or one whose elements share their storage, is refused whatever its size."""
    dev = torch.device("cuda", 0)
    for d in (dev, 0):
        for ws in (torch.empty(1 << 12, dtype=torch.uint8), torch.empty(1 << 12, dtype=torch.uint8, device="meta"), b"0" * 4096):
            with pytest.raises((ValueError, TypeError)):
                _lib._workspace(64, d, ws)
            with pytest.raises((ValueError, TypeError)):
                _lib._space(64, d, ws)
    assert _lib._space(0, 0, None) == (None, None, 0)


@pytest.mark.gpu
def test_workspaces_on_the_gpu():
    g = ref.gen(1)
    dy, w, r = ref.normal(g, 40, 64), ref.normal(g, 64), torch.ones(40, device="cuda:0")
    n = _lib.ft_rmsnorm_bwd_workspace_size(40, 64)
    whole = torch.empty(2 * n, dtype=torch.uint8, device="cuda:0")
    for ws in (whole[:1].expand(2 * n), whole[::2], torch.empty(n, dtype=torch.uint8), whole[:n - 16]):
        with pytest.raises(ValueError):
            _lib.ft_rmsnorm_bwd(dy, dy, w, r, workspace=ws)
    want = _lib.ft_rmsnorm_bwd(dy, dy, w, r)[1]
    for ws in (whole, whole[:n], whole[16:].view(torch.float32)):
        assert torch.equal(_lib.ft_rmsnorm_bwd(dy, dy, w, r, workspace=ws)[1], want)
