"""Cases of the 8-bit operators around the MXFP4 weights on one MI355X.

A layer keeps its frozen weight in MXFP4 (codes [N, K / 2], one power-of-two
scale per 32 x 32 tile) and takes its activations and gradients in MXFP8: E4M3
values with one power-of-two scale per 32 elements of a row, the smallest one
with which none of the 32 passes 448.  Scales lie as [K / 128, M, 4], rounded
up: block 4 g + j of row m at [g, m, j], and 1 past the row's end.

Kinds:
  norm        h = x + residual, y = h / rms(h) * w, and y in MXFP8 (and, in
              training, y in bf16 and 1 / rms in fp32)
  norm_bwd    its gradients: dx (of x and of the residual) and dw
  quant       a matrix in MXFP8: with its product with the low-rank factor, or
              a gradient on its way through an activation, dy * act'(z)
  linear      y = act(X W^T + P U + bias) + residual (and, in training, the
              activation's input z)
  linear_bwd  dx = (G W + Q D^T) * act'(z) + residual

`run` with `own` false is the plain form in torch; `exact` is the definition in
64 bits.
"""
import math

import torch

own = False

DEV = "cuda:0"
BF, F32, F64, U8, F8, E8 = (torch.bfloat16, torch.float32, torch.float64, torch.uint8, torch.float8_e4m3fn,
                            torch.float8_e8m0fnu)
EPS = 1e-6
ACTS = ("none", "gelu", "silu", "relu")
#: Products of the largest layer, which no drawn one passes.
MOST = 18432 * 4096 * 16384


def _norm(name, M, K, residual, train):
    c = {"kind": "norm", "M": M, "K": K, "residual": residual, "train": train}
    return dict(c, name=name) if name else c


def _norm_bwd(name, M, K, dh):
    c = {"kind": "norm_bwd", "M": M, "K": K, "dh": dh}
    return dict(c, name=name) if name else c


def _quant(name, M, K, R, by_r, act):
    c = {"kind": "quant", "M": M, "K": K, "R": R, "by_r": by_r, "act": act}
    return dict(c, name=name) if name else c


def _linear(name, M, K, N, R, act, residual, train=False, out="bf16"):
    c = {"kind": "linear", "M": M, "K": K, "N": N, "R": R, "act": act, "residual": residual, "train": train, "out": out}
    return dict(c, name=name) if name else c


def _linear_bwd(name, M, K, N, R, act, residual, out="bf16"):
    c = {"kind": "linear_bwd", "M": M, "K": K, "N": N, "R": R, "act": act, "residual": residual, "out": out}
    return dict(c, name=name) if name else c


def listed():
    return [
        # one new token of one sequence: the norm between two layers, where launches and latency are all
        _norm("norm_token", 1, 4096, True, False),
        # a training step's tokens: y and 1 / rms are kept for the backward
        _norm("norm_train", 4608, 4096, True, True),
        # the norm's gradients: a training step's tokens, and a width and a count that fit no tile
        _norm_bwd("norm_bwd_train", 4608, 4096, True),
        _norm_bwd("norm_bwd_ragged", 1111, 2080, False),
        # attention's output before its projection, with X [L1 | A] of the layer's low-rank branches
        _quant("quant_lora", 4608, 4096, 64, False, "none"),
        # the gradient on its way into an activated layer that has none of them
        _quant("quant_act_grad", 1111, 11264, 0, False, "silu"),
        # decoding, one sequence and sixteen: output projection into the residual stream, and the wide layer
        _linear("linear_token", 1, 4096, 4096, 32, "none", True),
        _linear("linear_tokens16", 16, 4096, 16384, 32, "silu", False),
        # the wide layer over a training step's tokens, and the largest: four times as many
        _linear("linear_train", 4608, 4096, 16384, 64, "gelu", False, train=True),
        _linear("linear_prefill", 18432, 4096, 16384, 0, "silu", False),
        # its input gradient, through the activation in front of it
        _linear_bwd("linear_bwd_train", 4608, 16384, 4096, 64, "gelu", False),
        # a short sequence through a layer of odd widths, result and residual in 32 bits
        _linear_bwd("linear_bwd_ragged_f32", 333, 2080, 3168, 48, "none", True, out="f32"),
    ]


def _log(rng, lo, hi):
    return math.exp(rng.uniform(math.log(lo), math.log(hi)))


def _width(rng, lo, hi):
    """A layer width: a multiple of 128 mostly (what models have), else of 32."""
    m = 128 if rng.random() < 0.7 else 32
    return max(m, int(round(_log(rng, lo, hi) / m)) * m)


def draw(rng):
    kind = rng.choice(["norm", "norm_bwd", "quant", "linear", "linear", "linear_bwd"])
    M = int(_log(rng, 1, 18433))
    if kind == "norm":
        return _norm(None, M, _width(rng, 256, 8192), rng.random() < 0.7, rng.random() < 0.5)
    if kind == "norm_bwd":
        return _norm_bwd(None, M, _width(rng, 256, 8192), rng.random() < 0.7)
    if kind == "quant":
        if rng.random() < 0.5:
            return _quant(None, M, _width(rng, 256, 16384), 16 * rng.randint(1, 6), rng.random() < 0.5, "none")
        return _quant(None, M, _width(rng, 256, 16384), 0, False, rng.choice(ACTS))
    while True:
        K, N = _width(rng, 256, 16384), _width(rng, 256, 16384)
        if M * K * N <= MOST:
            break
        M = int(_log(rng, 1, 18433))
    R, act, residual = 16 * rng.choice([0, 1, 2, 2, 4, 6]), rng.choice(ACTS), rng.random() < 0.5
    out = "f32" if rng.random() < 0.2 else "bf16"
    if kind == "linear":
        return _linear(None, M, K, N, R, act, residual, act != "none" and rng.random() < 0.5, out)
    return _linear_bwd(None, M, K, N, R, act, residual, out)


# ------------------------------------------------------------------- inputs
def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed) * 7919 + 29)
    return g


def _normal(g, shape, std=1.0):
    return torch.randn(shape, generator=g, device=DEV) * std


def _activations(g, M, K):
    """N(0, 1) with 0.5 % outlier channels x30."""
    x = _normal(g, (M, K))
    x[:, torch.randperm(K, generator=g, device=DEV)[:max(1, round(0.005 * K))]] *= 30.0
    return x.to(BF)


def _gradient(g, M, N):
    """Heavy-tailed: 1e-3 * Student-t with three degrees of freedom."""
    chi = torch.zeros((M, N), device=DEV)
    for _ in range(3):
        chi += _normal(g, (M, N)) ** 2
    return (1e-3 * _normal(g, (M, N)) / torch.sqrt(chi / 3.0)).to(BF)


def _weight(g, N, K):
    """N(0, 0.02^2) in MXFP4: codes [N, K / 2], scales [N / 32, K / 32]."""
    t = _normal(g, (N // 32, 32, K // 32, 32), 0.02)
    e = torch.frexp(t.abs().amax((1, 3), keepdim=True))[1] - 3
    t = t * _pow2(127 - e)
    code = torch.bucketize(t.abs(), torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0], device=DEV)).to(U8)
    code = (code | (t < 0).to(U8) << 3).reshape(N, K)
    return code[:, 0::2] | code[:, 1::2] << 4, (e.reshape(N // 32, K // 32) + 127).to(U8)


def _prepared(case, seed):
    """The inputs, and the buffers that a program keeps for the outputs."""
    g, kind, M, K = _gen(seed), case["kind"], case["M"], case["K"]
    buf = lambda *shape, t=BF: torch.empty(shape, dtype=t, device=DEV)  # noqa: E731
    codes = lambda C: {"codes": buf(M, C, t=F8), "scales": buf(-(-C // 128), M, 4, t=U8)}  # noqa: E731
    s = {"case": case}
    if kind == "norm":
        s.update(x=_normal(g, (M, K)).to(BF), w=(1.0 + _normal(g, (K,), 0.1)).to(BF),
                 residual=_activations(g, M, K) if case["residual"] else None, **codes(K))
        if case["residual"]:
            s["h"] = buf(M, K)
        if case["train"]:
            s.update(y=buf(M, K), rstd=buf(M, t=F32))
    elif kind == "norm_bwd":
        h = _activations(g, M, K)
        s.update(h=h, w=(1.0 + _normal(g, (K,), 0.1)).to(BF), dy=_gradient(g, M, K),
                 dh=_gradient(g, M, K) if case["dh"] else None,
                 rstd=torch.rsqrt(h.float().pow(2).mean(1) + EPS), dx=buf(M, K), dw=buf(K, t=F32))
    elif kind == "quant":
        R = case["R"]
        s.update(src=_activations(g, M, K) if R and not case["by_r"] else _gradient(g, M, K), **codes(K))
        if R:
            s.update(proj=_normal(g, (R, K) if case["by_r"] else (K, R), 0.01).to(BF), P=buf(M, R, t=F32))
        elif case["act"] != "none":
            s.update(z=_normal(g, (M, K)).to(BF), v=buf(M, K))
    else:
        N, R = case["N"], case["R"]
        back = kind == "linear_bwd"
        i, o = (N, K) if back else (K, N)          # the reduction's width, the result's
        t = F32 if case["out"] == "f32" else BF
        wq, ws = _weight(g, N, K)
        xq, xs = _mxfp8((_gradient if back else _activations)(g, M, i).float())
        s.update(wq=wq, ws=ws, xq=xq, xs=xs, P=None, F=None, bias=None, residual=None, out=buf(M, o, t=t))
        if R:
            s.update(P=_normal(g, (M, R), 0.02 if back else 1.0), F=_normal(g, (K, R) if back else (R, N), 0.01).to(BF))
        if not back:
            s["bias"] = _normal(g, (N,), 0.02).to(BF)
        if case["residual"]:
            s["residual"] = _normal(g, (M, o), 1e-3 if back else 1.0).to(t)
        if back and case["act"] != "none":
            s["z"] = _normal(g, (M, o)).to(BF)
        elif not back and case["train"]:
            s["z"] = buf(M, o)
    return s


def prepare(case, seed):
    return _prepared(case, seed)


# --------------------------------------------------------------- plain forms
def _pow2(code):
    """2^(code - 127) of codes 0 to 254, exactly."""
    return torch.where(code > 0, code.int() << 23, 1 << 22).view(F32)


def _mxfp8(y):
    """y fp32 [M, K] in MXFP8: E4M3 values [M, K] and the scales' bytes [K / 128, M, 4]."""
    M, K = y.shape
    t = y.unflatten(1, (-1, 32))
    bits = t.abs().amax(2).view(torch.int32)
    # the largest magnitude is m 2^E, 1 <= m < 2: E - 8, and one more where m passes 1.75 (448 = 1.75 2^8)
    code = ((bits >> 23) - 8 + ((bits & 0x7FFFFF) > 0x600000).int()).clamp(min=0)
    q = (t * _pow2(254 - code.unsqueeze(2))).to(F8).reshape(M, K)
    b = K // 32
    s = torch.full((M, -(-b // 4) * 4), 127, dtype=U8, device=y.device)
    s[:, :b] = code.to(U8)
    return q, s.unflatten(1, (-1, 4)).transpose(0, 1).contiguous()


def _values(q, s):
    """What E4M3 values [M, K] and the scales' bytes [K / 128, M, 4] stand for, fp32 [M, K]."""
    M, K = q.shape
    return (q.float().unflatten(1, (-1, 32)) * _pow2(s.transpose(0, 1).reshape(M, -1)[:, :K // 32, None])).flatten(1)


def _weights(wq, ws):
    """The weight's values, fp32 [N, K]."""
    lut = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6, -0.0, -0.5, -1, -1.5, -2, -3, -4, -6], device=DEV)
    w = lut[torch.stack([wq & 15, wq >> 4], 2).flatten(1).int()]
    N, K = w.shape
    return (w.view(N // 32, 32, K // 32, 32) * _pow2(ws)[:, None, :, None]).view(N, K)


def _act(a, z):
    if a == "gelu":
        return 0.5 * z * (1.0 + torch.tanh(math.sqrt(2.0 / math.pi) * (z + 0.044715 * z * z * z)))
    return z * torch.sigmoid(z) if a == "silu" else z.clamp(min=0.0) if a == "relu" else z


def _act_grad(a, z):
    if a == "gelu":
        c = math.sqrt(2.0 / math.pi)
        t = torch.tanh(c * (z + 0.044715 * z * z * z))
        return 0.5 * (1.0 + t) + 0.5 * z * (1.0 - t * t) * c * (1.0 + 3 * 0.044715 * z * z)
    if a == "silu":
        r = torch.sigmoid(z)
        return r + z * r * (1.0 - r)
    return (z > 0).to(z.dtype) if a == "relu" else torch.ones_like(z)


def run(s):
    c = s["case"]
    return (_own if own else _plain)[c["kind"]](s, c)


def _plain_norm(s, c):
    h = s["x"] if s["residual"] is None else (s["x"].float() + s["residual"].float()).to(BF)
    hf = h.float()
    rstd = torch.rsqrt(hf.pow(2).mean(1, keepdim=True) + EPS)
    y = hf * rstd * s["w"].float()
    q, sc = _mxfp8(y)
    out = {"codes": q, "scales": sc.view(E8)}
    if s["residual"] is not None:
        out["h"] = h
    if c["train"]:
        out.update(y=y.to(BF), rstd=rstd.flatten())
    return out


def _plain_norm_bwd(s, c):
    dy, r = s["dy"].float(), s["rstd"][:, None]
    xh = s["h"].float() * r
    g = dy * s["w"].float()
    dx = r * (g - xh * (g * xh).mean(1, keepdim=True))
    if s["dh"] is not None:
        dx = dx + s["dh"].float()
    return {"dx": dx.to(BF), "dw": (dy * xh).sum(0)}


def _plain_quant(s, c):
    y, out = s["src"].float(), {}
    if c["R"]:
        out["P"] = y @ (s["proj"].float().T if c["by_r"] else s["proj"].float())
    elif c["act"] != "none":
        y = y * _act_grad(c["act"], s["z"].float())
        out["v"] = y.to(BF)
    q, sc = _mxfp8(y)
    return dict(out, codes=q, scales=sc.view(E8))


def _plain_linear(s, c):
    z = _values(s["xq"], s["xs"]) @ _weights(s["wq"], s["ws"]).T + s["bias"].float()
    if c["R"]:
        z = z + s["P"] @ s["F"].float()
    y = _act(c["act"], z)
    if c["residual"]:
        y = y + s["residual"].float()
    out = {"y": y.to(s["out"].dtype)}
    return dict(out, z=z.to(BF)) if c["train"] else out


def _plain_linear_bwd(s, c):
    d = _values(s["xq"], s["xs"]) @ _weights(s["wq"], s["ws"])
    if c["R"]:
        d = d + s["P"] @ s["F"].float().T
    if c["act"] != "none":
        d = d * _act_grad(c["act"], s["z"].float())
    if c["residual"]:
        d = d + s["residual"].float()
    return {"dx": d.to(s["out"].dtype)}


_plain = {"norm": _plain_norm, "norm_bwd": _plain_norm_bwd, "quant": _plain_quant, "linear": _plain_linear,
          "linear_bwd": _plain_linear_bwd}


# ------------------------------------------------- the framework's operators
def _lib():
    from paper_2607_05711_amd import _lib
    return _lib


def _own_norm(s, c):
    _lib().ft_rmsnorm_quantize8(s["x"], s["w"], s["residual"], eps=EPS, h=s.get("h"), y=s.get("y"), codes=s["codes"],
                                scales=s["scales"], rstd=s.get("rstd"))
    out = {"codes": s["codes"], "scales": s["scales"].view(E8)}
    out.update((k, s[k]) for k in ("h", "y", "rstd") if k in s)
    return out


def _own_norm_bwd(s, c):
    _lib().ft_rmsnorm_bwd(s["dy"], s["h"], s["w"], s["rstd"], dh=s["dh"], dx=s["dx"], dw=s["dw"])
    return {"dx": s["dx"], "dw": s["dw"]}


def _own_quant(s, c):
    L = _lib()
    out = {"codes": s["codes"], "scales": s["scales"].view(E8)}
    if c["R"]:
        L.ft_quantize8(s["src"], proj=s["proj"], proj_layout=L.FT_PROJ_R_BY_COLS if c["by_r"] else L.FT_PROJ_COLS_BY_R,
                       codes=s["codes"], scales=s["scales"], proj_out=s["P"])
        return dict(out, P=s["P"])
    if c["act"] == "none":
        L.ft_quantize8(s["src"], codes=s["codes"], scales=s["scales"])
        return out
    L.ft_quantize8(s["src"], z=s["z"], act=ACTS.index(c["act"]), v=s["v"], codes=s["codes"], scales=s["scales"])
    return dict(out, v=s["v"])


def _own_linear(s, c):
    _lib().ft_linear8_fwd(s["xq"], s["xs"], s["wq"], s["ws"], s["P"], s["F"], s["bias"], act=ACTS.index(c["act"]),
                          residual=s["residual"], z=s.get("z"), y=s["out"])
    return {"y": s["out"], "z": s["z"]} if c["train"] else {"y": s["out"]}


def _own_linear_bwd(s, c):
    _lib().ft_linear8_bwd_input(s["xq"], s["xs"], s["wq"], s["ws"], s["P"], s["F"], z=s.get("z"),
                                act=ACTS.index(c["act"]), residual=s["residual"], dx=s["out"])
    return {"dx": s["out"]}


_own = {"norm": _own_norm, "norm_bwd": _own_norm_bwd, "quant": _own_quant, "linear": _own_linear,
        "linear_bwd": _own_linear_bwd}


# ----------------------------------------------------------- what it takes
def work(case):
    M, K, kind = case["M"], case["K"], case["kind"]
    if kind == "norm":
        b = M * K * (2 + 1 + 1 / 32) + 2 * K
        b += 2 * 2 * M * K if case["residual"] else 0
        b += M * (2 * K + 4) if case["train"] else 0
        return {"bytes": b, "flops": 6.0 * M * K}
    if kind == "norm_bwd":
        return {"bytes": M * K * (8 if case["dh"] else 6) + 4 * M + 6 * K, "flops": 12.0 * M * K}
    if kind == "quant":
        R, act = case["R"], case["act"] != "none"
        return {"bytes": M * K * (2 + 1 + 1 / 32 + (4 if act else 0)) + 2 * R * K + 4 * M * R,
                "flops": 2.0 * M * K * R + 2.0 * M * K}
    N, R, back = case["N"], case["R"], kind == "linear_bwd"
    i, o = (N, K) if back else (K, N)
    t = 4 if case["out"] == "f32" else 2
    b = N * K * (0.5 + 1 / 1024) + M * i * (1 + 1 / 32) + R * (4 * M + 2 * o) + M * o * t * (2 if case["residual"] else 1)
    b += 0 if back else 2 * N
    b += 2 * M * o if (case["act"] != "none" if back else case["train"]) else 0
    return {"bytes": b, "flops": 2.0 * M * N * K + 2.0 * M * R * o}


# -------------------------------------------------------------------- 64 bits
def _scale64(t):
    """log2 of the scale of each 32 elements: the smallest power of two that brings the largest to 448 = 7/8 2^9 or less."""
    f, e = torch.frexp(t.abs().amax(-1, keepdim=True))
    return torch.where(f > 0, e - 9 + (f > 0.875).int(), -127).clamp(min=-127)


def _codes64(y):
    """y over its blocks' scales, not rounded, and the scales."""
    M, K = y.shape
    t = y.unflatten(1, (-1, 32))
    e = _scale64(t)
    pad = -(K // 32) % 4
    s = torch.cat([torch.pow(2.0, e[..., 0].double()), torch.ones((M, pad), dtype=F64, device=y.device)], 1)
    return (t * torch.pow(2.0, -e.double())).flatten(1), s.view(M, -1, 4).permute(1, 0, 2).contiguous()


def _weights64(wq, ws):
    c = torch.empty((wq.shape[0], 2 * wq.shape[1]), dtype=torch.int64, device=DEV)
    c[:, 0::2], c[:, 1::2] = wq & 15, wq >> 4
    m, e = c & 1, c >> 1 & 3                            # E2M1: exponent bias 1, one mantissa bit
    v = torch.where(e > 0, (1.0 + 0.5 * m.double()) * torch.pow(2.0, e.double() - 1.0), 0.5 * m.double())
    s = torch.pow(2.0, ws.double() - 127.0).repeat_interleave(32, 0).repeat_interleave(32, 1)
    return torch.where(c > 7, -v, v) * s


def _values64(q, s):
    v = torch.pow(2.0, s.double() - 127.0).permute(1, 0, 2).flatten(1).repeat_interleave(32, 1)
    return q.double() * v[:, :q.shape[1]]


def _act64(a, z):
    if a == "gelu":
        return torch.nn.functional.gelu(z, approximate="tanh")
    return torch.nn.functional.silu(z) if a == "silu" else torch.relu(z) if a == "relu" else z


def _act_grad64(a, z):
    with torch.enable_grad():
        z = z.detach().requires_grad_(True)
        return torch.autograd.grad(_act64(a, z).sum(), z)[0]


def exact(case, seed):
    s, kind = _prepared(case, seed), case["kind"]
    d = {k: v.double() for k, v in s.items() if isinstance(v, torch.Tensor) and v.is_floating_point() and v.dtype != F8}
    if kind == "norm":
        h = d["x"] + d["residual"] if case["residual"] else d["x"]
        n = h.to(BF).double() if case["residual"] else h          # the stored stream is what is normed
        rstd = 1.0 / torch.sqrt((n * n).mean(1, keepdim=True) + EPS)
        y = n * rstd * d["w"]
        q, sc = _codes64(y)
        out = {"codes": q, "scales": sc}
        if case["residual"]:
            out["h"] = h
        return dict(out, y=y, rstd=rstd[:, 0]) if case["train"] else out
    if kind == "norm_bwd":
        with torch.enable_grad():
            h, w = (d[k].requires_grad_(True) for k in ("h", "w"))
            y = h * torch.rsqrt((h * h).mean(1, keepdim=True) + EPS) * w
            dx, dw = torch.autograd.grad(y, (h, w), d["dy"])
        return {"dx": dx + d["dh"] if case["dh"] else dx, "dw": dw}
    if kind == "quant":
        y, out = d["src"], {}
        if case["R"]:
            out["P"] = torch.einsum("mk,rk->mr", y, d["proj"]) if case["by_r"] else torch.einsum("mk,kr->mr", y, d["proj"])
        elif case["act"] != "none":
            y = out["v"] = y * _act_grad64(case["act"], d["z"])
        q, sc = _codes64(y)
        return dict(out, codes=q, scales=sc)
    x, w = _values64(s["xq"], s["xs"]), _weights64(s["wq"], s["ws"])
    if kind == "linear":
        z = torch.addmm(d["bias"], x, w.T)
        z = torch.addmm(z, d["P"], d["F"]) if case["R"] else z
        y = _act64(case["act"], z) + (d["residual"] if case["residual"] else 0.0)
        return {"y": y, "z": z} if case["train"] else {"y": y}
    dx = torch.mm(x, w)
    dx = torch.addmm(dx, d["P"], d["F"].T) if case["R"] else dx
    dx = dx * _act_grad64(case["act"], d["z"]) if case["act"] != "none" else dx
    return {"dx": dx + d["residual"] if case["residual"] else dx}
