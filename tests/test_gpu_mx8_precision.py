"""What the 8-bit linear's results owe to the matrix instruction, and what they do not depend on."""
import ctypes

import pytest
import torch

from tests import _mx8 as ref
from tests._mx8 import BF, F32, F64, F8, U8
from paper_2607_05711_amd import _lib as L

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.fixture
def on_tile(monkeypatch):
    """Sends the linear's calls to the kernel with this output tile (1: of few rows)."""
    def use(tile):
        lib, launch, to = L.load(), L._launch, {}
        for n in ("ft_linear8_fwd", "ft_linear8_bwd_input"):
            f = getattr(lib, n.replace("ft_", "ftx_"))
            f.argtypes, f.restype = [ctypes.c_int] + getattr(lib, n).argtypes, ctypes.c_int
            to[n] = f
        monkeypatch.setattr(L, "_launch", lambda f, dev, *a: launch(to[f.__name__], dev, tile, *a))
    return use


def operands(g, M, K, N, back, outliers):
    """A quantized activation (or gradient) with channels x30 where asked for, a quantized weight, both in 64 bits."""
    x = ref.normal(g, M, N if back else K)
    if outliers:
        x[:, 3::200] *= 30
    wq, ws, _ = L.ft_quantize_blockwise(ref.normal(g, N, K, std=0.02), block_rows=32)
    xq, xs, _, _ = L.ft_quantize8(x)
    W = ref.values4(wq, ws)
    return xq, xs, wq, ws, ref.values8(xq, xs), W if back else W.T.contiguous()


def exponents(X, W):
    """Exponents of E4M3 and E2M1 values over their scales, subnormals with their format's least (X: codes, W: values)."""
    return torch.frexp(X)[1].clamp(min=-5) - 1, torch.frexp(W)[1].clamp(min=1) - 1


def lost(xq, wq, X, W, back):
    """Per element of the product, what groups of eight may drop: (sum, root of the sum of squares).

    In a group what lies below 2^-14 of the largest product's power of two is dropped, so a product loses less than
    2^(E - 13), whether E is the exponent of the largest product or the largest sum of two factors' exponents, one
    less than it where the significands carry; and nothing if it is a multiple of that."""
    M, K = X.shape
    N = W.shape[1]
    x = ref.values8(xq, torch.full(((K + 127) // 128, M, 4), 127, dtype=U8, device=DEV))
    one = torch.full((wq.shape[0] // 32 * (wq.shape[1] // 16),), 127, dtype=U8, device=DEV)
    w = ref.values4(wq, one)
    w = w if back else w.T.contiguous()
    ex, ew = exponents(x, w)
    total, square = torch.zeros((M, N), dtype=F64, device=DEV), torch.zeros((M, N), dtype=F64, device=DEV)
    for k in range(0, K, 8):
        p = x[:, k:k + 8, None] * w[None, k:k + 8]
        e = torch.where(p != 0, ex[:, k:k + 8, None] + ew[None, k:k + 8], -100).amax(1, keepdim=True)
        e = torch.maximum(e, torch.frexp(p.abs().amax(1, keepdim=True))[1] - 1)
        u = ref.pow2(e - 13)
        n = (p != torch.round(p / u) * u).sum(1)
        # the scales are the group's own: X's of 32 elements, W's of a 32 x 32 tile
        s = torch.where(x[:, k:k + 8] != 0, X[:, k:k + 8] / x[:, k:k + 8], 0).amax(1)[:, None] * \
            torch.where(w[k:k + 8] != 0, W[k:k + 8] / w[k:k + 8], 0).amax(0)[None]
        u = u[:, 0] * s
        total += n * u
        square += n * u * u
    return total, square.sqrt()


@pytest.mark.parametrize("outliers", [False, True])
@pytest.mark.parametrize("back", [False, True])
@pytest.mark.parametrize("tile", [64, 128, 192, 256])
def test_what_product_groups_drop(tile, back, outliers, on_tile):
    """bf16 results, seen before their rounding: a residual takes most of each away, and what is left is rounded at its
    own, smaller size (half a step: 2^-8 of it).

    Every element is off by at most what its groups drop (lost) and K / 8 roundings of partial sums to fp32; in the
    2-norm the groups' losses, of random signs, add by their squares."""
    M, K, N = (200, 1024, 96) if not back else (200, 96, 1024)
    xq, xs, wq, ws, X, W = operands(ref.gen(tile + back), M, K, N, back, outliers)
    on_tile(tile)
    want = X @ W
    r = (-want).to(BF)
    f = L.ft_linear8_bwd_input if back else L.ft_linear8_fwd
    y = f(xq, xs, wq, ws, residual=r).double()
    total, rms = lost(xq, wq, X, W, back)
    left = want + r.double()
    S = X.abs() @ W.abs()
    fp32 = (1024 / 8 + 2) * 2.0 ** -24 * S
    off = (y - left).abs()
    tol = (total + fp32) * (1 + 2.0 ** -8) + left.abs() * 2.0 ** -8
    assert bool((off <= tol).all()), float((off / tol).max())
    # (partial sums of random terms are on average no larger than the whole; twice their roundings' share)
    assert float(off.norm()) <= float(rms.norm() + (1024 / 8 + 2) ** 0.5 * 2.0 ** -23 * want.norm() + left.norm() * 2.0 ** -8)
    # and fp32 results, whose groups are exact
    exact = f(xq, xs, wq, ws, out_dtype=F32).double()
    assert bool(((exact - want).abs() <= 2 * fp32 + want.abs() * 2.0 ** -24).all())


@pytest.mark.parametrize("f32,act,residual,R", [(False, 0, False, 0), (False, 1, True, 48), (True, 2, True, 32), (True, 3, False, 16)])
@pytest.mark.parametrize("back", [False, True])
@pytest.mark.parametrize("tile", [1, 64, 128, 192, 256])
def test_rows_do_not_depend_on_their_neighbours(tile, back, f32, act, residual, R, on_tile):
    """On one kernel a row's bits are the same whatever rows stand beside it and wherever in a tile it is."""
    if tile == 1 and back:
        pytest.skip("the kernel of few rows: forward")
    on_tile(tile)
    g = ref.gen(tile + R)
    M, (K, N) = 32 if tile == 1 else 600, (672, 288) if not back else (288, 672)
    i, o = (N, K) if back else (K, N)
    xq, xs = ref.operand(g, M, i)
    wq, ws = ref.weight(g, N, K)
    P = ref.normal(g, M, R, dtype=F32) if R else None
    F = ref.normal(g, *((K, R) if back else (R, N))) if R else None
    res = ref.normal(g, M, o, dtype=F32 if f32 else BF) if residual else None
    z = ref.normal(g, M, o) if back and act else None
    b = None if back else ref.normal(g, N)

    def call(rows):
        cut = lambda t: None if t is None else t[rows].contiguous()  # noqa: E731
        a = (cut(xq.view(U8)).view(F8), xs[:, rows].contiguous(), wq, ws, cut(P), F)
        kw = dict(act=act, residual=cut(res), out_dtype=F32 if f32 else BF)
        return L.ft_linear8_bwd_input(*a, z=cut(z), **kw) if back else L.ft_linear8_fwd(*a, b, **kw)
    every = call(torch.arange(M, device=DEV))
    # (on 64 x 128 tiles both sizes are shared by two groups of waves: at most 256 tiles)
    for rows in (torch.arange(M // 2 - 3, device=DEV), torch.arange(1, device=DEV) + M - 1,
                 torch.randperm(M, generator=g, device=DEV)[:M - 5]):
        assert torch.equal(call(rows).view(U8), every[rows].view(U8))


@pytest.mark.parametrize("M", [1, 40, 700])
def test_norm_codes_into_the_linear(M):
    """A layer without adapters behind the norm takes its codes as they are; one with adapters takes P from y."""
    g = ref.gen(M)
    K, N, R = 416, 288, 32
    x, res, w = ref.normal(g, M, K), ref.normal(g, M, K), 1 + ref.normal(g, K, std=0.1)
    wq, ws, _ = L.ft_quantize_blockwise(ref.normal(g, N, K, std=0.05), block_rows=32)
    D, U, b = ref.normal(g, K, R, std=K ** -0.5), ref.normal(g, R, N, std=0.1), ref.normal(g, N, std=0.1)
    h, y, c, s, _ = L.ft_rmsnorm_quantize8(x, w, res, want_y=True)
    P = L.ft_quantize8(y, proj=D)[2]
    out = L.ft_linear8_fwd(c, s, wq, ws, bias=b, act=L.FT_ACT_SILU, out_dtype=F32)
    low = L.ft_linear8_fwd(c, s, wq, ws, P, U, b, act=L.FT_ACT_SILU, out_dtype=F32)
    h64, _, y64 = ref.norm64(x, res, w, 1e-6)
    assert torch.equal(h.double(), h64)
    W = ref.values4(wq, ws).T
    # the codes' own values: fp32 results, exact groups, K / 4 roundings of partial sums
    V = ref.values8(c, s)
    for got, extra, mag in ((out, 0.0, 0.0), (low, P.double() @ U.double(), P.double().abs() @ U.double().abs())):
        a = V @ W + extra + b.double()
        S = V.abs() @ W.abs() + mag + b.double().abs()
        tol = (K / 4 + R + 8) * 2.0 ** -24 * S
        want = ref.act64(2, a)
        tol = tol * 1.2 + ref.act_slack(a) * a.abs().clamp(max=1) + want.abs() * 2.0 ** -23
        assert bool(((got.double() - want).abs() <= tol).all())
    # and the norm's: an E4M3 rounding is off by at most half a step, 2^-4 of the value, or 2^-10 of the block's scale
    e = ref.pow2(s.transpose(0, 1).reshape(M, -1)[:, :K // 32].int() - 127).repeat_interleave(32, 1)
    slack = (y64.abs() * (2.0 ** -4 + 2.0 ** -18) + 2.0 ** -10 * e) @ W.abs()
    a64 = y64 @ W + b.double()
    # (SiLU' is at most 1.1 in size)
    assert bool(((out.double() - ref.act64(2, a64)).abs() <= 1.1 * slack + 2.0 ** -16 * (1 + a64.abs())).all())
