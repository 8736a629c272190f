"""Measured calls of the training operators around the widely-linear layers:
layer norm (or RMSNorm) with the residual addition and its backward pass, the
8-bit form of activations and gradients, and the product of two 8-bit matrices.

A case is a dict of plain values; ``kind`` selects the operator:

norm       x, delta complex64 [B, n] -> h = x + delta, the norm of its 2n reals
           (mean taken off where ``center``), (mean, 1/sigma) of each token; the
           norm in bf16, or where ``fp8`` in 8 bits (returned as the values).
norm_grad  the norm's gradient: dz bf16 [B, n, 2] and the residual's dh -> dx,
           and the gradients of gain and bias, summed over the tokens.
quantise   a matrix of reals -> its 8-bit form along the rows, along the columns
           (transposed) or both, as ``form`` says, returned as the values.
gemm       C = A B^T of two 8-bit matrices, C in bf16.
wgrad      a layer's weight gradient G_Y^T X from the 8-bit activations kept by
           the forward pass and the bf16 gradient G_Y of its output.

8-bit form of a matrix [rows, cols]: e4m3 codes [rows, cp], cp = cols rounded
up to 128 (zeros there), and a byte e + 127 for each 128 neighbours of a row,
uint8 [ceil(cols / 512), rows, 4] (four blocks of a row side by side).  A code
stands for its value times 2^e; e is the smallest with max |x| <= 448 * 2^e,
within [-117, 119].  Rounding is to nearest, ties to even.
"""
import math
import random

import torch

own = False

MAX_FLOPS = 2 * 4096 * 4096 * 11008  # the largest listed product
MAX_NORM = 4096 * 2048               # tokens x entries of the largest listed norm
MAX_CELLS = 4096 * 11008             # reals of the largest listed quantisation


def listed():
    return [
        # one token between two layers: launch and host latency
        dict(name="norm_b1", kind="norm", B=1, n=2048, center=True, delta=True, fp8=False),
        # a ragged batch of a width that no power of two divides (3000 reals), RMSNorm
        dict(name="norm_odd_b77", kind="norm", B=77, n=1500, center=False, delta=True, fp8=False),
        # the norm in front of a layer's 8-bit product in a step of 4096 tokens of a 4096-wide model
        dict(name="norm_fp8_4096", kind="norm", B=4096, n=2048, center=True, delta=True, fp8=True),
        # its backward pass for a few tokens of a narrow model: latency
        dict(name="norm_grad_b5", kind="norm_grad", B=5, n=257, center=True, dh=False),
        # and for the whole step, RMSNorm, the residual's gradient added
        dict(name="norm_grad_4096", kind="norm_grad", B=4096, n=2048, center=False, dh=True),
        # odd sizes, both forms, float32 input that is part of a wider array
        dict(name="quantise_odd", kind="quantise", rows=509, cols=3002, dtype="float32", form="both", wide=True),
        # a layer's real form for the forward product and the input's gradient
        dict(name="quantise_gate", kind="quantise", rows=11008, cols=4096, dtype="bfloat16", form="both", wide=False),
        # a few tokens through a narrow layer: latency
        dict(name="gemm_b16", kind="gemm", M=16, N=512, K=512),
        # odd sizes in every direction, the last tiles of all axes ragged
        dict(name="gemm_odd", kind="gemm", M=1003, N=2750, K=1378),
        # the down projection's forward product, 4096 tokens
        dict(name="gemm_down_4096", kind="gemm", M=4096, N=4096, K=11008),
        # an odd layer's weight gradient over a ragged number of tokens
        dict(name="wgrad_odd", kind="wgrad", M=1003, N=1378, K=2750),
        # the square layer's weight gradient, 4096 tokens: gradient and checkpoint turned, product; in bf16, as
        # gradients that are reduced over ranks are
        dict(name="wgrad_q_4096", kind="wgrad", M=4096, N=4096, K=4096),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    while True:
        kind = rng.choice(("norm", "norm_grad", "quantise", "gemm", "gemm", "wgrad"))
        if kind in ("norm", "norm_grad"):
            case = dict(kind=kind, B=_log(rng, 1, 8192), n=_log(rng, 16, 8192), center=rng.random() < 0.5)
            if kind == "norm":
                case.update(delta=rng.random() < 0.8, fp8=rng.random() < 0.5)
            else:
                case.update(dh=rng.random() < 0.7)
            if case["B"] * case["n"] <= MAX_NORM:
                return case
        elif kind == "quantise":
            case = dict(kind=kind, rows=_log(rng, 1, 16384), cols=_log(rng, 1, 16384),
                        dtype=rng.choice(("float32", "bfloat16")), form=rng.choice(("rows", "columns", "both")),
                        wide=rng.random() < 0.3)
            if case["rows"] * case["cols"] <= MAX_CELLS:
                return case
        else:
            case = dict(kind=kind, M=_log(rng, 1, 16384), N=_log(rng, 16, 16384), K=_log(rng, 16, 16384))
            if kind == "wgrad":  # rows of complex tokens: even numbers of reals
                case["N"] += case["N"] % 2
                case["K"] += case["K"] % 2
            if (2 * case["M"] * case["N"] * case["K"] <= MAX_FLOPS
                    and max(case["M"] * case["N"], case["M"] * case["K"], case["N"] * case["K"]) <= MAX_CELLS):
                return case


def work(case):
    kind = case["kind"]
    if kind == "norm":
        e = case["B"] * case["n"]
        # h is an output of its own only where something was added; the 8-bit form is written and read back
        return {"bytes": e * ((24 if case["delta"] else 8) + (8 if case["fp8"] else 4)) + 16 * case["n"]
                + 8 * case["B"], "flops": 16 * e}
    if kind == "norm_grad":
        e = case["B"] * case["n"]
        return {"bytes": e * (8 + 4 + 8 + (8 if case["dh"] else 0)) + 24 * case["n"] + 8 * case["B"], "flops": 32 * e}
    if kind == "quantise":
        e = case["rows"] * case["cols"]
        forms = 2 if case["form"] == "both" else 1
        return {"bytes": e * ((4 if case["dtype"] == "float32" else 2) + 4 * forms), "flops": 4 * e * forms}
    M, N, K = case["M"], case["N"], case["K"]
    if kind == "gemm":
        return {"bytes": M * K + N * K + 2 * M * N, "flops": 2 * M * N * K}
    # both operands are read, written in their turned form and read again
    return {"bytes": M * N * (2 + 2) + M * K * (1 + 2) + 2 * N * K, "flops": 2 * M * N * K}


# -------------------------------------------------------- the 8-bit form


def _scale_bytes(e, rows, cols):
    """Exponents [rows, blocks] -> bytes [ceil(cols / 512), rows, 4]."""
    nb = e.shape[1]
    s = torch.nn.functional.pad((e + 127).to(torch.uint8), (0, -nb % 4))
    return s.reshape(rows, -1, 4).transpose(0, 1).contiguous()


def _power(e):
    """2^e in float32, exact, for e in [-126, 127] (pow and ldexp round on the GPU)."""
    return ((e.int() + 127) << 23).view(torch.float32)


def _quantise(x):
    """float32 [rows, cols] -> (codes, scale bytes, values in float32)."""
    rows, cols = x.shape
    nb = -(-cols // 128)
    blocks = torch.nn.functional.pad(x, (0, nb * 128 - cols)).reshape(rows, nb, 128)
    m, e = torch.frexp(blocks.abs().amax(-1))  # amax = m 2^e, m in [0.5, 1); 448 = 0.875 * 2^9
    e = torch.where(m == 0, -117, (e - 9 + (m > 0.875)).clamp(-117, 119))
    codes = (blocks * _power(-e)[..., None]).to(torch.float8_e4m3fn)
    values = (codes.float() * _power(e)[..., None]).reshape(rows, nb * 128)[:, :cols]
    return codes.reshape(rows, nb * 128), _scale_bytes(e, rows, cols), values


def _values(codes, scales, rows, cols):
    """Codes and scale bytes -> float32 [rows, cols]."""
    e = scales.transpose(0, 1).reshape(rows, -1)[:, :codes.shape[1] // 128].int() - 127
    return (codes.float().reshape(rows, -1, 128) * _power(e)[..., None]).reshape(rows, -1)[:, :cols]


# ------------------------------------------------------------------ prepare


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)

    def normal(*shape):
        return torch.randn(shape, generator=g, device="cuda")

    kind, s = case["kind"], dict(case=case)
    if kind in ("norm", "norm_grad"):
        B, n = case["B"], case["n"]
        spread = torch.exp(normal(1, n, 1))  # a residual stream's channels differ in size
        s["gain"] = 1 + 0.1 * normal(2 * n)
        s["bias"] = 0.1 * normal(2 * n) if case["center"] else None
        x = normal(B, n, 2) * spread
        if kind == "norm":
            s["x"] = torch.view_as_complex(x)
            s["delta"] = torch.view_as_complex(0.3 * normal(B, n, 2)) if case["delta"] else None
            return s
        mu = x.double().mean((1, 2)) if case["center"] else torch.zeros(B, dtype=torch.float64, device="cuda")
        r = ((x.double() - mu[:, None, None]).square().mean((1, 2)) + 1e-5).rsqrt()
        s["h"], s["stats"] = torch.view_as_complex(x), torch.stack([mu, r], 1).float().contiguous()
        s["dz"] = (0.01 * normal(B, n, 2)).to(torch.bfloat16)
        s["dh"] = torch.view_as_complex(0.01 * normal(B, n, 2)) if case["dh"] else None
        return s
    if kind == "quantise":
        rows, cols = case["rows"], case["cols"]
        # a gradient's or a weight's rows differ in size, and so do its columns
        x = normal(rows, cols + 22 if case["wide"] else cols) * torch.exp(normal(rows, 1))
        x = x[:, 11:11 + cols] if case["wide"] else x
        x.mul_(torch.exp(0.5 * normal(1, cols)))
        s["x"] = x if case["dtype"] == "float32" else x.to(torch.bfloat16)
        if case["wide"] and case["dtype"] == "bfloat16":
            s["x"] = torch.nn.functional.pad(s["x"], (11, 11))[:, 11:11 + cols]
        return s
    M, N, K = case["M"], case["N"], case["K"]
    a = normal(M, K) * torch.exp(0.5 * normal(1, K))  # activations: channels that stand out
    s["a"] = _quantise(a)[:2]
    if kind == "gemm":
        s["b"] = _quantise(0.02 * normal(N, K))[:2]
    else:
        s["gy"] = (0.001 * normal(M, N) * torch.exp(0.5 * normal(M, 1))).to(torch.bfloat16).reshape(M, N // 2, 2)
    return s


# ---------------------------------------------------------------- plain form


def _plain_norm(s):
    case = s["case"]
    h = s["x"] if s["delta"] is None else s["x"] + s["delta"]
    r = torch.view_as_real(h)
    B, n = h.shape
    mu = r.sum((1, 2)) / (2 * n) if case["center"] else torch.zeros(B, device="cuda")
    c = r - mu[:, None, None]
    inv = torch.rsqrt(c.square().sum((1, 2)) / (2 * n) + 1e-5)
    z = c * inv[:, None, None] * s["gain"].reshape(2, n).t()
    if s["bias"] is not None:
        z = z + s["bias"].reshape(2, n).t()
    if case["fp8"]:
        z = _quantise(z.reshape(B, 2 * n))[2].reshape(B, n, 2)
    return {"h": h, "z": z.to(torch.bfloat16), "stats": torch.stack([mu, inv], 1)}


def _plain_norm_grad(s):
    case = s["case"]
    h, dz = torch.view_as_real(s["h"]), s["dz"].float()
    B, n = s["h"].shape
    mu, r = (s["stats"][:, i, None, None] for i in (0, 1))
    xh = (h - mu) * r
    w = dz * s["gain"].reshape(2, n).t()
    t = xh * ((w * xh).sum((1, 2), keepdim=True) / (2 * n))
    if case["center"]:
        t = t + w.sum((1, 2), keepdim=True) / (2 * n)
    dx = (w - t) * r
    if s["dh"] is not None:
        dx = dx + torch.view_as_real(s["dh"])
    out = {"dx": torch.view_as_complex(dx), "dgain": (dz * xh).sum(0).t().reshape(2 * n)}
    if case["center"]:
        out["dbias"] = dz.sum(0).t().reshape(2 * n)
    return out


def _plain_quantise(s):
    x, form = s["x"].float(), s["case"]["form"]
    out = {}
    if form != "columns":
        out["rows"] = _quantise(x)[2].to(torch.bfloat16)
    if form != "rows":
        out["columns"] = _quantise(x.t().contiguous())[2].to(torch.bfloat16)
    return out


def _plain_gemm(s):
    case = s["case"]
    a = _values(*s["a"], case["M"], case["K"])
    b = _values(*s["b"], case["N"], case["K"])
    return torch.matmul(a, b.t()).to(torch.bfloat16)


def _plain_wgrad(s):
    case = s["case"]
    M, N, K = case["M"], case["N"], case["K"]
    x = _quantise(_values(*s["a"], M, K).t().contiguous())[2]
    g = _quantise(s["gy"].float().reshape(M, N).t().contiguous())[2]
    return torch.matmul(g, x.t()).to(torch.bfloat16)


# ----------------------------------------------------------------------- run


def _own(s):
    import paper_2512_02901_amd as f2
    case = s["case"]
    kind = case["kind"]
    if kind == "norm":
        h, z, stats = f2.add_layernorm(s["x"], s["gain"], bias=s["bias"], delta=s["delta"], eps=1e-5,
                                       center=case["center"], fp8=case["fp8"])
        return {"h": h, "z": z.dequantize().view(case["B"], case["n"], 2) if case["fp8"] else z, "stats": stats}
    if kind == "norm_grad":
        dx, dgain, dbias = f2.layernorm_backward(s["dz"], s["h"], s["stats"], s["gain"], dh=s["dh"],
                                                 center=case["center"], bias=case["center"])
        return {"dx": dx, "dgain": dgain, "dbias": dbias} if case["center"] else {"dx": dx, "dgain": dgain}
    if kind == "quantise":
        form = case["form"]
        if form == "both":
            direct, turned = f2.quantize_fp8(s["x"], transposed="both")
            return {"rows": direct.dequantize(), "columns": turned.dequantize()}
        return {form: f2.quantize_fp8(s["x"], transposed=form == "columns").dequantize()}
    if "A" not in s:
        s["A"] = f2.Fp8Matrix(case["M"], case["K"], *s["a"])
    if kind == "gemm":
        if "B" not in s:
            s["B"] = f2.Fp8Matrix(case["N"], case["K"], *s["b"])
        return f2.gemm_fp8(s["A"], s["B"])
    return f2.gemm_fp8(f2.quantize_fp8(s["gy"], transposed=True), s["A"].transpose())


def run(state):
    if own:
        return _own(state)
    return {"norm": _plain_norm, "norm_grad": _plain_norm_grad, "quantise": _plain_quantise, "gemm": _plain_gemm,
            "wgrad": _plain_wgrad}[state["case"]["kind"]](state)


# --------------------------------------------------------------------- exact


def _exact_blocks(x):
    """float64 [rows, cols] -> what its 8-bit form stands for: each value's nearest of e4m3 times the block's power of two."""
    out = torch.empty_like(x)
    for at in range(0, x.shape[1], 128):
        b = x[:, at:at + 128]
        top = b.abs().amax(1, keepdim=True)
        unit = torch.exp2(torch.ceil(torch.log2(top / 448)).clamp(-117, 119))
        # log2 may be off beside a power of two
        unit = torch.where(top > 448 * unit, 2 * unit, unit)
        unit = torch.where((top <= 224 * unit) & (unit > 2.0 ** -117), unit / 2, unit)
        u = (b / unit).abs()
        # the grid's step is 2^-3 of a value's power of two, 2^-9 below 2^-6
        step = torch.exp2(torch.frexp(u.clamp(min=2.0 ** -6))[1].double() - 4)
        out[:, at:at + 128] = torch.round(u / step) * step * unit * torch.sign(b)
    return out


def _exact_values(codes, scales, rows, cols):
    b = codes.view(torch.uint8).long()
    e, m = b >> 3 & 15, (b & 7).double()
    v = torch.where(e > 0, (8 + m) * torch.exp2(e.double() - 10), m * 2.0 ** -9) * (1 - 2 * (b >> 7)).double()
    for k in range(codes.shape[1] // 128):
        v[:, 128 * k:128 * (k + 1)] *= torch.exp2(scales[k // 4, :, k % 4].double() - 127)[:, None]
    return v[:, :cols]


def _exact_norm(s):
    case = s["case"]
    x = s["x"].to(torch.complex128)
    if s["delta"] is not None:
        x = x + s["delta"].to(torch.complex128)
    B, n = x.shape
    flat = torch.cat([x.real, x.imag], 1)  # the layer's real vector, [Re x ; Im x]
    mu = flat.mean(1) if case["center"] else torch.zeros(B, dtype=torch.float64, device="cuda")
    dev = torch.sqrt(((flat - mu[:, None]) ** 2).mean(1) + 1e-5)
    z = (flat - mu[:, None]) / dev[:, None] * s["gain"].double()
    if s["bias"] is not None:
        z += s["bias"].double()
    z = torch.stack([z[:, :n], z[:, n:]], 2)
    if case["fp8"]:
        z = _exact_blocks(z.reshape(B, 2 * n)).reshape(B, n, 2)
    return {"h": x, "z": z, "stats": torch.stack([mu, 1 / dev], 1)}


def _exact_norm_grad(s):
    case = s["case"]
    n = case["n"]
    flat = torch.cat([s["h"].real, s["h"].imag], 1).double()
    dz = torch.cat([s["dz"][..., 0], s["dz"][..., 1]], 1).double()
    mean, r = s["stats"].double()[:, :1], s["stats"].double()[:, 1:]
    y = (flat - mean) * r
    # the Jacobian of the norm is r (I - y y^T / 2n - 1 1^T / 2n), with the last part where the mean is taken off
    w = dz * s["gain"].double()
    dx = w - y * (w * y).mean(1, keepdim=True)
    if case["center"]:
        dx -= w.mean(1, keepdim=True)
    dx = torch.complex(*(r * dx).split(n, 1))
    if s["dh"] is not None:
        dx += s["dh"].to(torch.complex128)
    out = {"dx": dx, "dgain": (dz * y).sum(0)}
    if case["center"]:
        out["dbias"] = dz.sum(0)
    return out


def exact(case, seed):
    s = prepare(case, seed)
    kind = case["kind"]
    if kind == "norm":
        return _exact_norm(s)
    if kind == "norm_grad":
        return _exact_norm_grad(s)
    if kind == "quantise":
        x = s["x"].double()
        out = {}
        if case["form"] != "columns":
            out["rows"] = _exact_blocks(x)
        if case["form"] != "rows":
            out["columns"] = _exact_blocks(x.t().contiguous())
        return out
    M, N, K = case["M"], case["N"], case["K"]
    a = _exact_values(*s["a"], M, K)
    if kind == "gemm":
        return a @ _exact_values(*s["b"], N, K).t().contiguous()
    g = s["gy"].double().reshape(M, N).t().contiguous()
    return _exact_blocks(g) @ _exact_blocks(a.t().contiguous()).t().contiguous()
