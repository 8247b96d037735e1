"""MXFP8 references for the tests, in 64 bits: the E4M3 table and the block rule
written from their definitions, and the 8-bit linear's operands."""
import torch

BF, F32, F64, U8, F8 = torch.bfloat16, torch.float32, torch.float64, torch.uint8, torch.float8_e4m3fn


def e4m3_values():
    """Magnitudes of codes 0 to 126 (bias 7, subnormals in steps of 2^-9)."""
    c = torch.arange(127, dtype=torch.int64)
    e, m = c >> 3, (c & 7).double()
    return torch.where(e > 0, (1 + m / 8) * pow2(e - 7), m / 8 * 2.0 ** -6)


def pow2(e):
    return ((e.to(torch.int64) + 1023) << 52).view(F64)


def block_scale(t):
    """Code of the smallest e >= -127 with max|t| <= 448 2^e over the last dimension (t fp64, finite)."""
    a = t.abs().amax(-1)
    f, e = torch.frexp(a)                                     # a = f 2^e, 1/2 <= f < 1; 448 = 7/8 2^9
    e = torch.where(a > 0, e - 9 + (f > 0.875), torch.full_like(e, -127)).clamp(min=-127)
    return (e + 127).to(U8)


def mxfp8(x):
    """(codes uint8 [M, K], scales uint8 [ceil(K / 128), M, 4]) of x [M, K] (any float type), by nearest search on the
    table of magnitudes, ties to the even code."""
    M, K = x.shape
    t = x.double().unflatten(1, (-1, 32))
    s = block_scale(t)
    a = (t / pow2(s.int() - 127)[..., None]).abs()
    v = e4m3_values().to(x.device)
    hi = torch.searchsorted(v, a).clamp(max=126)              # first value >= a
    lo = (hi - 1).clamp(min=0)
    dh, dl = v[hi] - a, a - v[lo]
    code = torch.where((dl < dh) | ((dl == dh) & (lo % 2 == 0)), lo, hi)
    sign = (torch.signbit(t).to(torch.int64) << 7)
    pad = torch.full((M, -(K // 32) % 4), 127, dtype=U8, device=x.device)
    scales = torch.cat([s, pad], 1).unflatten(1, (-1, 4)).transpose(0, 1).contiguous()
    return (code | sign).to(U8).flatten(1), scales


def values8(codes, scales):
    """What codes (float8_e4m3fn) and scales stand for, fp64 [M, K]."""
    M, K = codes.shape
    c = codes.view(U8).to(torch.int64)
    v = e4m3_values().to(codes.device)[(c & 127).clamp(max=126)]
    v = torch.where((c & 127) == 127, torch.nan, v)
    v = torch.where(c > 127, -v, v)
    b = scales.transpose(0, 1).reshape(M, -1)[:, :K // 32].int()
    s = torch.where(b == 255, torch.nan, pow2(b - 127))
    return (v.unflatten(1, (-1, 32)) * s[..., None]).flatten(1)


def values4(wq, ws):
    """The weight's values, fp64 [N, K]."""
    mag = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6], dtype=F64, device=wq.device)
    c = torch.stack([wq & 15, wq >> 4], -1).flatten(1).long()
    N, K = c.shape
    s = pow2(ws.reshape(N // 32, K // 32).int() - 127).repeat_interleave(32, 0).repeat_interleave(32, 1)
    return torch.where(c > 7, -mag[c & 7], mag[c & 7]) * s


def act64(a, z):
    if a == 1:
        return torch.nn.functional.gelu(z, approximate="tanh")
    return torch.nn.functional.silu(z) if a == 2 else torch.relu(z) if a == 3 else z


def act_grad64(a, z):
    """act'(z), from the closed forms."""
    if a == 1:
        c = (2.0 / torch.pi) ** 0.5
        t = torch.tanh(c * (z + 0.044715 * z ** 3))
        return 0.5 * (1 + t) + 0.5 * z * (1 - t * t) * c * (1 + 3 * 0.044715 * z * z)
    if a == 2:
        r = torch.sigmoid(z)
        return r + z * r * (1 - r)
    return (z > 0).double() if a == 3 else torch.ones_like(z)


def act_slack(z):
    """Error of act(z) and act'(z) in fp32 on the hardware's exp2 and reciprocal.  The exponent's argument, of size
    up to 2|z| (and c z^3 for the GELU, where |z| > 5 has long saturated), is off by 2^-23 of itself, exp2 and
    reciprocal by 2^-23 each, and at most four more roundings follow, on values of size at most 1.2 (1 + |z|): some
    ten units of 2^-24 (1 + |z|)."""
    return 2.0 ** -20 * (1 + z.abs())


def norm64(x, residual, w, eps):
    """(h as stored, rstd, y) in fp64."""
    h = x.double() if residual is None else (x.float() + residual.float()).to(BF).double()
    rstd = 1 / torch.sqrt((h * h).mean(1) + eps)
    return h, rstd, h * rstd[:, None] * w.double()


def norm_bwd64(dy, h, w, rstd, dh):
    dy, h, w, r = dy.double(), h.double(), w.double(), rstd.double()[:, None]
    n, g = h * r, dy * w
    dx = r * (g - n * (g * n).mean(1, keepdim=True))
    return (dx if dh is None else dx + dh.double()), (dy * n).sum(0)


def normal(g, *shape, std=1.0, dtype=BF):
    return (torch.randn(shape, generator=g, device=g.device) * std).to(dtype)


def weight(g, N, K):
    """Codes and tile scales of a random weight: every code, scales 2^-9 to 2^-3."""
    wq = torch.randint(0, 256, (N, K // 2), dtype=U8, device=g.device, generator=g)
    ws = torch.randint(118, 125, (N // 32, K // 32), dtype=U8, device=g.device, generator=g)
    return wq, ws


def operand(g, M, K):
    """MXFP8 operand of random codes (no NaN) and scales 2^-4 to 2^4; pad scales hold NaN codes, which are not read."""
    c = torch.randint(0, 127, (M, K), device=g.device, generator=g).to(U8)
    c = c | (torch.randint(0, 2, (M, K), device=g.device, generator=g).to(U8) << 7)
    G = (K + 127) // 128
    s = torch.randint(123, 132, (G, M, 4), dtype=U8, device=g.device, generator=g)
    if K % 128:
        s[-1, :, K % 128 // 32:] = 255
    return c.view(F8), s


def gen(seed, device="cuda:0"):
    g = torch.Generator(device=device)
    g.manual_seed(seed)
    return g
