"""Quantisation, norms and 4-bit products from their definitions, in numpy on the CPU (FP32 where the definition rounds, FP64 elsewhere)."""
import numpy as np
import torch

from paper_2511_10909_b200 import workloads as wl

U = 2.0 ** -24                              # half a step of FP32, relative
FORMATS = ["e4m3", "e5m2", "mxe4m3", "mxe5m2", "mxf4", "nvf4"]
TOP = {"e4m3": 448.0, "e5m2": 57344.0, "e2m1": 6.0}
EMAX = {"mxe4m3": 8, "mxe5m2": 15, "mxf4": 2}
BLOCK = {"mxe4m3": 32, "mxe5m2": 32, "mxf4": 32, "nvf4": 16}
DTYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}
HALF_STEP = {k: torch.finfo(t).eps / 2 for k, t in DTYPES.items()}      # of a rounding, relative


def elem(fmt):
    return wl.elem_format(fmt)


def blocks(y, fmt):
    kb = BLOCK[fmt]
    M, K = y.shape
    return np.pad(y, ((0, 0), (0, -K % kb))).reshape(M, -1, kb)


def e8m0(amax, fmt):
    """Codes of non-negative finite amax."""
    e = np.frexp(amax)[1].astype(np.int64) - 1
    return np.where(amax == 0, 0, np.clip(e - EMAX[fmt] + 127, 0, 254)).astype(np.uint8)


def quantize(x, fmt):
    """float32 matrix -> (codes, sf, row_scale) as the library's definition has them; one code per byte for FP4 (see pack)."""
    x = np.asarray(x, dtype=np.float32)
    M, K = x.shape
    f32 = np.float32
    with np.errstate(all="ignore"):
        if fmt in ("e4m3", "e5m2"):
            bad = ~np.isfinite(x).all(1)
            s = np.maximum(np.abs(x).max(1) / f32(TOP[fmt]), f32(2.0 ** -126)).astype(f32)
            codes = wl.cast_small(np.where(bad[:, None], 0, x / s[:, None]), fmt)
            codes[bad] = 0x7F
            s[bad] = np.nan
            return codes, None, s
        b = blocks(x, fmt)
        amax = np.abs(b).max(2)
        if fmt == "nvf4":
            bad = ~np.isfinite(x).all(1)
            s = np.maximum(np.abs(x).max(1) / f32(2688.0), f32(2.0 ** -100)).astype(f32)
            ratio = amax / (f32(6.0) * s)[:, None]
            ratio[bad] = 0
            g = np.maximum(wl.cast_small(ratio, "ue4m3"), 1)
            t = wl.small_values(g.astype(np.int64), "ue4m3").astype(f32) * s[:, None]
            q = b / t[:, :, None]
            q[bad] = 0
            codes = wl.cast_small(q, "e2m1").reshape(M, -1)[:, :K]
            codes[bad], g[bad], s[bad] = 0, 0x7F, np.nan
            return codes, g, s
        bad = ~np.isfinite(b).all(2)
        sf = e8m0(np.where(bad, 0, amax), fmt)
        q = np.ldexp(np.where(bad[:, :, None], 0, b), (127 - sf.astype(np.int64))[:, :, None].astype(np.int32))
        codes = wl.cast_small(q, elem(fmt))
        codes[bad] = 0 if fmt == "mxf4" else 0x7F
        sf[bad] = 255
        return codes.reshape(M, -1)[:, :K], sf, None


def pack(codes, fmt):
    return wl.pack_fp4(codes) if fmt in ("mxf4", "nvf4") else codes


def unpack(codes, fmt):
    if fmt not in ("mxf4", "nvf4"):
        return codes
    out = np.empty((codes.shape[0], codes.shape[1] * 2), np.uint8)
    out[:, 0::2], out[:, 1::2] = codes & 15, codes >> 4
    return out


def scale_values(sf, fmt):
    v = 2.0 ** (sf.astype(np.float64) - 127) if fmt != "nvf4" else wl.small_values(sf.astype(np.int64), "ue4m3").astype(np.float64)
    return np.where(sf == (0x7F if fmt == "nvf4" else 255), np.nan, v)


def code_values(codes, fmt):
    v = wl.small_values(codes.astype(np.int64), elem(fmt)).astype(np.float64)
    if elem(fmt) != "e2m1":
        m = codes & 0x7F
        v = np.where(m > (0x7E if elem(fmt) == "e4m3" else 0x7B), np.nan, v)
    return v


def units(q, fmt, K):
    """What one unit of every code stands for (M x K) under the scales of (codes, sf, row_scale)."""
    _, sf, s = q
    M = len(s) if s is not None else len(sf)
    u = np.ones((M, K))
    if sf is not None:
        u = np.repeat(scale_values(sf, fmt), BLOCK[fmt], axis=1)[:, :K]
    return u if s is None else u * s.astype(np.float64)[:, None]


def half_spacing(v, fmt):
    """Half the distance between the codes' values around v (magnitudes up to the largest)."""
    eb, mb, bias, _ = wl._SMALL[elem(fmt)]
    e = np.maximum(np.frexp(np.abs(v))[1] - 1, 1 - bias)
    return np.ldexp(0.5, e - mb)


def assert_quantised(q, y, fmt, rel):
    """(codes, sf, row_scale) against 64-bit y that the kernel knows to `rel` relative: the scales are what the definition says but for that
    error, and every code is one nearest to y / scale but for it."""
    codes, sf, s = q
    M, K = y.shape
    if s is not None:
        want = np.maximum(np.abs(y).max(1) / (2688.0 if fmt == "nvf4" else TOP[fmt]), 2.0 ** (-100 if fmt == "nvf4" else -126))
        assert (np.abs(s - want) <= (rel + 2 * U) * want).all()
    if fmt in EMAX:
        b = np.abs(blocks(y, fmt)).max(2)
        lo, hi = e8m0(b * (1 - rel), fmt), e8m0(b * (1 + rel), fmt)
        assert ((sf == lo) | (sf == hi)).all()
    if fmt == "nvf4":
        ratio = np.abs(blocks(y, fmt)).max(2) / (6.0 * s.astype(np.float64)[:, None])
        lo, hi = (np.maximum(wl.cast_small(ratio * (1 + d * (rel + 4 * U)), "ue4m3"), 1) for d in (-1, 1))
        assert ((sf >= lo) & (sf <= hi)).all()
    v = code_values(codes, fmt)
    want = y / units(q, fmt, K)
    want = np.clip(want, -TOP[elem(fmt)], TOP[elem(fmt)])
    err = np.abs(v - want)
    assert (err <= half_spacing(np.maximum(np.abs(v), np.abs(want)), fmt) + (rel + 4 * U) * np.abs(want)).all(), err.max()


# relative error of the norm before its last rounding: a sum of K squares by threads of up to 64 elements and a tree over up to 512 threads
# (at most 64 + 10 roundings on its way, and the square root halves them), the division by K, eps, the root, two products
NORM_REL = ((64 + 10) / 2 + 6) * U


def rms_norm(h, w, eps):
    """y in 64 bits, and 1 / rms."""
    r = 1.0 / np.sqrt((h * h).mean(1, keepdims=True) + eps)
    return h * r * (1.0 if w is None else w), r


def rms_norm_backward(dy, h, w, res, eps):
    """(dx, dweight, error bounds of both before their last rounding), from 64-bit inputs.

    Bounds: r is known to (37 + 6) U, so r g to 46 U; c = r^3 / K sum(g h) to 3 x 43 + 8 roundings and the sum's own 74 U of its terms'
    magnitudes; dweight adds M products known to 45 U in some order."""
    K, M = h.shape[1], h.shape[0]
    g = dy if w is None else dy * w
    _, r = rms_norm(h, None, eps)
    c = r ** 3 / K * (g * h).sum(1, keepdims=True)
    dx = r * g - h * c + (0.0 if res is None else res)
    mag = r ** 3 / K * np.abs(g * h).sum(1, keepdims=True)
    bound = U * (48 * np.abs(r * g) + np.abs(h) * (140 * np.abs(c) + 78 * mag) + 3 * np.abs(dx) + (0.0 if res is None else 2 * np.abs(res)))
    return dx, (dy * h * r).sum(0), bound, U * (M + 50) * np.abs(dy * h * r).sum(0)


def weights(codes, sf, fmt, row_scale=None):
    """Unpacked FP4 codes and scales -> 64-bit weights."""
    v = code_values(codes, fmt)
    with np.errstate(invalid="ignore"):
        v = v * np.repeat(scale_values(sf, fmt), BLOCK[fmt], axis=1)
        return v if row_scale is None else v * row_scale.astype(np.float64)[:, None]


def matvec_bound(x, w, K):
    """Error before the last rounding: sums of 128 products by eight instructions, each of which truncates 17 terms 2^-24 below the largest,
    then additions in FP32 (K / 1024 of them by a warp, eight warps, three parts, scale)."""
    return (8 * 18 + K / 1024 + 16) * U * (np.abs(x) @ np.abs(w).T)
