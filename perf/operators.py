"""The operators around matrix products of scaled 8- and 4-bit operands, as cases that can be timed and compared.

  quantize   mmasim.quantize: a matrix into codes and scales as mmasim.gemm takes them
  norm       mmasim.rms_norm: root-mean-square norm with the residual's addition, its output plain or quantised
  backward   mmasim.rms_norm_backward: the norm's gradients
  matvec     mmasim.matvec4: the product of a few tokens with 4-bit weights and group scales

With `own` false every operator is computed by elementary torch operations in FP32.  Codes come back as the values that they stand
for: FP8 as float8 tensors, FP4 as float8 tensors of the same values.
"""
import math

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
BYTES = {"bf16": 2, "fp16": 2, "fp32": 4}
FP8 = {"e4m3": (torch.float8_e4m3fn, 448.0), "e5m2": (torch.float8_e5m2, 57344.0)}
EMAX = {"mxe4m3": 8, "mxe5m2": 15, "mxf4": 2}
BLOCK = {"mxe4m3": 32, "mxe5m2": 32, "mxf4": 32, "nvf4": 16}
FORMATS = ["e4m3", "e5m2", "mxe4m3", "mxe5m2", "mxf4", "nvf4"]
EPS = 1e-6
TINY = {"e4m3": 2.0 ** -126, "e5m2": 2.0 ** -126, "nvf4": 2.0 ** -100}


def _case(op, M, K, dtype, **kw):
    return dict(op=op, M=M, K=K, dtype=dtype, **kw)


def listed():
    return [
        # the norm in front of a projection while one sequence is generated: nothing but latency
        dict(_case("norm", 1, 4096, "bf16", fmt="e4m3", residual=True, wide=False), name="norm_token_e4m3"),
        # the same over a prompt, block-scaled output
        dict(_case("norm", 4096, 4096, "bf16", fmt="mxe4m3", residual=True, wide=False), name="norm_prompt_mxfp8"),
        # sizes that nobody chose with vectors in mind, plain output
        dict(_case("norm", 1000, 1111, "fp16", fmt="", residual=True, wide=True), name="norm_ragged_fp16"),
        # a whole batch of training rows, row scales
        dict(_case("norm", 16384, 8192, "bf16", fmt="e4m3", residual=True, wide=False), name="norm_batch_e4m3"),
        # the gradients of a small batch, and of one in FP32 with odd sizes
        dict(_case("backward", 4096, 4096, "bf16", residual=True, wide=False), name="backward_4096"),
        dict(_case("backward", 777, 1111, "fp32", residual=False, wide=False), name="backward_ragged_fp32"),
        # a weight matrix into group-scaled FP4
        dict(_case("quantize", 4096, 4096, "bf16", fmt="nvf4"), name="quantize_nvf4_weights"),
        # activations of a large layer into FP8 with row scales
        dict(_case("quantize", 2048, 14336, "fp16", fmt="e5m2"), name="quantize_e5m2_rows"),
        # one token through a square projection
        dict(_case("matvec", 1, 4096, "bf16", N=4096, fmt="nvf4"), name="matvec_token_4096"),
        # one token through a wide layer: the stream of the weights alone counts
        dict(_case("matvec", 1, 8192, "bf16", N=28672, fmt="nvf4"), name="matvec_token_28672"),
        # a handful of sequences at once
        dict(_case("matvec", 8, 4096, "fp16", N=14336, fmt="mxf4"), name="matvec_batch_8"),
        # odd numbers of outputs and of blocks, FP32 activations
        dict(_case("matvec", 3, 4128, "fp32", N=1111, fmt="mxf4"), name="matvec_ragged_fp32"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _up(x, to):
    return -(-x // to) * to


def draw(rng):
    op = rng.choices(["norm", "backward", "quantize", "matvec"], [3, 2, 2, 3])[0]
    dtype = rng.choice(["bf16", "bf16", "fp16", "fp32"])
    if op == "matvec":
        T, N, K = _log(rng, 1, 16), _log(rng, 16, 28672), _up(_log(rng, 32, 16384), 32)
        while N * K > 1 << 27:
            N, K = -(-N // 2), _up(-(-K // 2), 32)
        if rng.random() < 0.5:
            N, K = _up(N, 16), _up(K, 128)
        return _case(op, T, K, dtype, N=N, fmt=rng.choice(["mxf4", "nvf4"]))
    M, K = _log(rng, 1, 16384), _log(rng, 64, 16384)
    while M * K * BYTES[dtype] > 1 << 27:
        M = -(-M // 2)
    if rng.random() < 0.5:              # half of the sizes as networks have them, half as they come
        K = _up(K, 64)
    if op == "backward":
        return _case(op, M, K, dtype, residual=rng.random() < 0.5, wide=rng.random() < 0.3)
    fmt = rng.choice(FORMATS if op == "quantize" else FORMATS[:4] + ["", "", "nvf4"])
    if fmt in ("mxf4", "nvf4"):
        K = _up(K, 32)
    if op == "quantize":
        return _case(op, M, K, dtype, fmt=fmt)
    return _case(op, M, K, dtype, fmt=fmt, residual=rng.random() < 0.6, wide=rng.random() < 0.3)


# ---- inputs, made on the GPU ----
def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)

    def normal(*shape):
        return torch.randn(shape, generator=gen, device="cuda")

    M, K, dt = case["M"], case["K"], DTYPES[case["dtype"]]
    s = {"case": case}
    if case["op"] == "matvec":
        w = normal(case["N"], K) * (1.5 / math.sqrt(K))
        s["W"], s["sf"], s["row_scale"] = _packed(w, case["fmt"])
        s["x"] = normal(M, K).to(dt)
        return s
    # activations: most features near one, a few in a hundred an order of magnitude larger
    feature = torch.where(torch.rand((1, K), generator=gen, device="cuda") < 0.02, 12.0, 1.0)
    s["x"] = (normal(M, K) * feature).to(dt)
    if case["op"] == "quantize":
        return s
    s["weight"] = (1.0 + 0.1 * normal(K)).to(torch.float32 if case["wide"] else dt)
    if case["op"] == "backward":
        s["dy"] = (normal(M, K) * 0.01).to(dt)
    s["residual"] = (normal(M, K) * (0.01 if case["op"] == "backward" else 2.0)).to(dt) if case["residual"] else None
    return s


def _packed(w, fmt):
    """A matrix of weights as a checkpoint holds it: two codes per byte, scale bytes, FP32 row scales (NVFP4)."""
    q = _quantize(w, fmt)
    v = q["codes"].float()
    code = torch.bucketize(v.abs(), torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0], device=v.device)) + 8 * (v < 0)
    code = code.to(torch.uint8)
    return (code[:, 0::2] | (code[:, 1::2] << 4)).contiguous(), q["sf"].view(torch.uint8), q.get("row_scale")


# ---- the plain forms ----
def _e2m1(q):
    a = q.abs()
    mag = 0.5 * ((a > 0.25).float() + (a >= 0.75).float() + (a > 1.25).float() + (a >= 1.75).float()) \
        + (a > 2.5).float() + (a >= 3.5).float() + 2.0 * (a > 5.0).float()
    return torch.where(q < 0, -mag, mag).to(torch.float8_e4m3fn)


def _blocks(y, kb):
    M, K = y.shape
    if K % kb:
        y = torch.cat([y, y.new_zeros(M, kb - K % kb)], 1)
    return y.view(M, -1, kb)


def _quantize(y, fmt):
    """FP32 matrix -> values of the codes, scales."""
    M, K = y.shape
    if fmt in FP8:
        kind, top = FP8[fmt]
        s = (y.abs().amax(1) / top).clamp_min(TINY[fmt])
        return {"codes": (y / s[:, None]).clamp(-top, top).to(kind), "row_scale": s}
    b = _blocks(y, BLOCK[fmt])
    amax = b.abs().amax(2)
    if fmt == "nvf4":
        s = (y.abs().amax(1) / 2688.0).clamp_min(TINY[fmt])
        g = (amax / (6.0 * s)[:, None]).clamp(2.0 ** -9, 448.0).to(torch.float8_e4m3fn)
        return {"codes": _e2m1((b / (g.float() * s[:, None])[:, :, None]).view(M, -1)[:, :K]), "sf": g, "row_scale": s}
    e = torch.where(amax > 0, torch.frexp(amax)[1] - 1 - EMAX[fmt], -127).clamp(-127, 127)
    q = torch.ldexp(b, -e[:, :, None]).view(M, -1)[:, :K]
    if fmt == "mxf4":
        codes = _e2m1(q)
    else:
        kind, top = FP8[fmt[2:]]
        codes = q.clamp(-top, top).to(kind)
    return {"codes": codes, "sf": (e + 127).to(torch.uint8).view(torch.float8_e8m0fnu)}


def _plain(s):
    c, x = s["case"], s["x"].float()
    if c["op"] == "quantize":
        return _quantize(x, c["fmt"])
    if c["op"] == "matvec":
        codes = torch.stack([s["W"] & 15, s["W"] >> 4], 2).view(c["N"], c["K"])
        value = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0, -0.0, -0.5, -1.0, -1.5, -2.0, -3.0, -4.0, -6.0], device=x.device)
        w = value[codes.int()]
        kind = torch.float8_e4m3fn if c["fmt"] == "nvf4" else torch.float8_e8m0fnu
        w = (w.view(c["N"], -1, BLOCK[c["fmt"]]) * s["sf"].view(kind).float()[:, :, None]).view(c["N"], c["K"])
        y = x @ w.t()
        if s["row_scale"] is not None:
            y = y * s["row_scale"]
        return y.to(s["x"].dtype)
    w = s["weight"].float()
    if c["op"] == "backward":
        dy = s["dy"].float()
        r = torch.rsqrt(x.square().mean(1, keepdim=True) + EPS)
        g = dy * w
        dx = r * g - x * (r * r * r / c["K"] * (g * x).sum(1, keepdim=True))
        if s["residual"] is not None:
            dx = dx + s["residual"].float()
        return {"dx": dx.to(s["x"].dtype), "dweight": (dy * x * r).sum(0).to(s["weight"].dtype)}
    out, h = {}, x
    if s["residual"] is not None:
        out["residual"] = (x + s["residual"].float()).to(s["x"].dtype)
        h = out["residual"].float()
    y = h * torch.rsqrt(h.square().mean(1, keepdim=True) + EPS) * w
    if c["fmt"]:
        out.update(_quantize(y, c["fmt"]))
    else:
        out["y"] = y.to(s["x"].dtype)
    return out


# ---- the framework's operators ----
_pairs = {}


def _fp4_values(codes):
    """Packed E2M1 codes -> the float8 tensor of their values (a table of the 256 bytes, two values each)."""
    if codes.device not in _pairs:
        v = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0, -0.0, -0.5, -1.0, -1.5, -2.0, -3.0, -4.0, -6.0], device=codes.device)
        v = v.to(torch.float8_e4m3fn).view(torch.uint8)
        byte = torch.arange(256, device=codes.device)
        _pairs[codes.device] = torch.stack([v[byte & 15], v[byte >> 4]], 1).contiguous().view(torch.int16).view(-1)
    return _pairs[codes.device][codes.int()].view(torch.float8_e4m3fn)


def _values(q, fmt):
    out = {}
    if fmt in ("mxf4", "nvf4"):
        out["codes"] = _fp4_values(q.codes)
    else:
        out["codes"] = q.codes.view(FP8[fmt[-4:]][0])
    if q.sf is not None:
        out["sf"] = q.sf.view(torch.float8_e4m3fn if fmt == "nvf4" else torch.float8_e8m0fnu)
    if q.row_scale is not None:
        out["row_scale"] = q.row_scale
    return out


def _own(s):
    from paper_2511_10909_b200 import mmasim
    c = s["case"]
    if c["op"] == "quantize":
        return _values(mmasim.quantize(s["x"], c["fmt"]), c["fmt"])
    if c["op"] == "matvec":
        return mmasim.matvec4(c["fmt"], s["W"], s["sf"], s["x"], s["row_scale"])
    if c["op"] == "backward":
        dx, dweight = mmasim.rms_norm_backward(s["dy"], s["x"], s["weight"], s["residual"], eps=EPS)
        return {"dx": dx, "dweight": dweight}
    y, residual = mmasim.rms_norm(s["x"], s["weight"], s["residual"], eps=EPS, fmt=c["fmt"] or None)
    out = _values(y, c["fmt"]) if c["fmt"] else {"y": y}
    if residual is not None:
        out["residual"] = residual
    return out


def run(state):
    return _own(state) if own else _plain(state)


# ---- the definitions in 64 bits ----
def _nearest(q, bits, low, top):
    """The nearest value with `bits` bits behind the leading one, exponents from `low` on, at most `top` (ties to even)."""
    step = torch.ldexp(torch.ones_like(q), (torch.frexp(q)[1] - 1).clamp_min(low) - bits)
    return (torch.round(q / step) * step).clamp(-top, top)


_GRID = {"e4m3": (3, -6, 448.0), "e5m2": (2, -14, 57344.0), "f4": (1, 0, 6.0)}


def _exact_codes(y, fmt):
    M, K = y.shape
    if fmt in FP8:
        s = torch.clamp(torch.max(torch.abs(y), dim=1).values / _GRID[fmt][2], min=2.0 ** -126)
        return {"codes": _nearest(y / s.unsqueeze(1), *_GRID[fmt]), "row_scale": s}
    kb = 16 if fmt == "nvf4" else 32
    n = (K + kb - 1) // kb
    wide = torch.zeros((M, n * kb), dtype=torch.float64, device=y.device)
    wide[:, :K] = y
    top = torch.abs(wide).reshape(M, n, kb).max(dim=2).values
    if fmt == "nvf4":
        s = torch.clamp(torch.max(torch.abs(y), dim=1).values / (448 * 6), min=2.0 ** -100)
        sf = torch.clamp(_nearest(top / (6 * s).unsqueeze(1), 3, -6, 448.0), min=2.0 ** -9)
        unit = sf * s.unsqueeze(1)
    else:
        sf = unit = torch.exp2(torch.clamp(torch.floor(torch.log2(top)) - EMAX[fmt], -127, 127))
        s = None
    q = _nearest((wide.reshape(M, n, kb) / unit.unsqueeze(2)).reshape(M, n * kb)[:, :K], *_GRID[fmt[-2:] if fmt in ("mxf4", "nvf4") else fmt[2:]])
    out = {"codes": q, "sf": sf}
    if s is not None:
        out["row_scale"] = s
    return out


def exact(case, seed):
    s = prepare(case, seed)
    x = s["x"].double()
    op, fmt, K = case["op"], case.get("fmt"), case["K"]
    if op == "quantize":
        return _exact_codes(x, fmt)
    if op == "matvec":
        y = torch.zeros((case["M"], case["N"]), dtype=torch.float64, device=x.device)
        value = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]
        sf = s["sf"].int()
        if fmt == "nvf4":
            field, mant = sf >> 3, (sf & 7).double()
            sf = torch.where(field == 0, mant * 2.0 ** -9, torch.ldexp(1 + mant / 8, field - 7))
        else:
            sf = torch.ldexp(torch.ones_like(sf, dtype=torch.float64), sf - 127)
        for n in range(0, case["N"], 2048):             # rows at a time: the weights in 64 bits are large
            byte = s["W"][n:n + 2048].long()
            w = torch.zeros((byte.shape[0], K), dtype=torch.float64, device=x.device)
            for half in (0, 1):
                nibble = (byte >> (4 * half)) & 15
                w[:, half::2] = torch.tensor(value + [-v for v in value], dtype=torch.float64, device=x.device)[nibble]
            w *= sf[n:n + 2048].repeat_interleave(K // sf.shape[1], dim=1)
            y[:, n:n + 2048] = (w @ x.t()).t()
        return y if s["row_scale"] is None else y * s["row_scale"].double()
    w = s["weight"].double()
    if op == "backward":
        g, r = s["dy"].double(), 1 / torch.sqrt((x * x).sum(1) / K + EPS)
        unit = x * r.unsqueeze(1)
        dx = ((g * w) - unit * ((g * w * unit).sum(1) / K).unsqueeze(1)) * r.unsqueeze(1)
        if s["residual"] is not None:
            dx += s["residual"].double()
        return {"dx": dx, "dweight": (g * unit).sum(0)}
    out, h = {}, x
    if s["residual"] is not None:
        out["residual"] = x + s["residual"].double()
        h = out["residual"].to(s["x"].dtype).double()   # the norm is taken of what is stored
    y = h / torch.sqrt((h * h).sum(1) / K + EPS).unsqueeze(1) * w
    if fmt:
        out.update(_exact_codes(y, fmt))
    else:
        out["y"] = y
    return out


def work(case):
    M, K, b = case["M"], case["K"], BYTES[case["dtype"]]
    fmt = case.get("fmt")
    if case["op"] == "matvec":
        N = case["N"]
        return {"bytes": N * K / 2 + N * K / BLOCK[fmt] + (4 * N if fmt == "nvf4" else 0) + M * K * b + M * N * b, "flops": 2.0 * M * N * K}
    wb = 4 if case.get("wide") else b
    if case["op"] == "backward":
        return {"bytes": M * K * b * (3 + case["residual"]) + 2 * K * wb, "flops": 12.0 * M * K}
    if fmt:
        out = M * K * (0.5 if fmt in ("mxf4", "nvf4") else 1.0) + (M * -(-K // BLOCK[fmt]) if fmt in BLOCK else 0) + (4 * M if fmt in TINY else 0)
    else:
        out = M * K * b
    if case["op"] == "quantize":
        return {"bytes": M * K * b + out, "flops": 4.0 * M * K}
    return {"bytes": M * K * b * (1 + 2 * case["residual"]) + K * wb + out, "flops": 8.0 * M * K}
