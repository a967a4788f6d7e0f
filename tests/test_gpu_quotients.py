"""Codes of quotients next to the middle between two FP32 numbers, of which one is a tie of the codes."""
import numpy as np
import pytest
import torch

import rows_ref as ref

pytestmark = pytest.mark.gpu
if torch.cuda.is_available():
    from paper_2511_10909_b200 import mmasim

ROW_FORMATS = ["e4m3", "e5m2", "nvf4"]


def same(x, fmt):
    q = mmasim.quantize(torch.from_numpy(x).cuda(), fmt)
    c, sf, s = (None if t is None else t.cpu().numpy() for t in q)
    codes, sf_want, s_want = ref.quantize(x, fmt)
    assert np.array_equal(s, s_want) and (sf is None or np.array_equal(sf, sf_want))
    bad = np.argwhere(ref.unpack(c, fmt) != codes)
    assert bad.size == 0, (fmt, len(bad), [(x[tuple(b)], s[b[0]], ref.unpack(c, fmt)[tuple(b)], codes[tuple(b)]) for b in bad[:4]])


@pytest.mark.parametrize("fmt", ["e4m3", "e5m2"])
def test_scales_of_24_ones(fmt):
    """A divisor of 24 ones: its quotient of a power of two lies 2^-25 of a unit above the middle between that power and the next FP32
    number, and for one power it is the tie between zero and the smallest code."""
    top = np.float32(ref.TOP[fmt])
    x = np.zeros((160, 64), np.float32)
    for row in range(160):
        s = np.float32(np.ldexp(2.0 - 2.0 ** -23, row - 57))
        most = np.float32(np.float64(top) * s)
        for m in (most, np.nextafter(most, np.float32(0)), np.nextafter(most, np.float32(np.inf))):
            if m / top == s:
                x[row, 0] = m
        assert x[row, 0] != 0
        for k in range(24):
            x[row, 16 + k] = np.ldexp(1.0, row - 57 - k) * (-1) ** k
            x[row, 40 + k] = np.ldexp(2.0 - 2.0 ** -23, row - 57 - k)
    same(x, fmt)


def test_block_scales_of_24_ones():
    """The same for NVFP4, whose divisor is a block's scale times the row's (no row's scale alone has 24 ones)."""
    ones, rows = np.float32(2.0 - 2.0 ** -23), []
    for gain in range(9, 16):               # eighths
        g = np.float32(gain / 8)
        s = np.float32(np.float64(ones) / g)
        for s in (s, np.nextafter(s, np.float32(0)), np.nextafter(s, np.float32(4))):
            most = np.float32(2688.0 * np.float64(s))
            fits = [m for m in (most, np.nextafter(most, np.float32(0)), np.nextafter(most, np.float32(1e9))) if m / np.float32(2688.0) == s]
            if g * s != ones or not fits:
                continue
            row = np.zeros(48, np.float32)
            row[0], row[16] = fits[0], np.float32(6.0) * ones
            for k in range(15):
                row[17 + k] = np.ldexp(1.0, 3 - k) * (-1) ** k
                row[33 + k] = np.ldexp(1.0, 3 - k)
            row[32] = row[16]
            rows += [row * np.float32(2.0 ** e) for e in (-40, 0, 60)]
    assert len(rows) >= 6
    same(np.pad(np.stack(rows), ((0, 0), (0, 16))), "nvf4")


def beside_ties(fraction_bits):
    """(divisor, dividend) mantissas whose quotient is within 64 / 2^25 of a unit from the middle between a tie of at most `fraction_bits`
    bits behind the leading one and one of its neighbours, as whole numbers of 24 bits."""
    pairs = set()
    for frac in range(1 << fraction_bits):
        tie = (1 << 23) + (frac << (23 - fraction_bits))
        for q in (tie - 1, tie):
            twice = 2 * q + 1 if q >= 1 << 23 else (1 << 25) - 1
            for bits in (22, 23, 24, 25):
                inverse = pow(twice, -1, 1 << bits)
                for d in range(-64, 65):
                    for s in range(d * inverse % (1 << bits), 1 << 24, 1 << bits):
                        x = (s * twice - d) >> bits
                        if s >= 1 << 23 and x << bits == s * twice - d and 1 << 23 <= x < 1 << 24:
                            pairs.add((s, x))
    return sorted(pairs)


@pytest.mark.parametrize("fmt", ROW_FORMATS)
def test_quotients_beside_ties(fmt):
    """Every such divisor as a row's scale (NVFP4: as the scale of a row whose blocks have scales of powers of two), every such dividend under it
    at all places of its exponent that matter."""
    pairs = [p for p in beside_ties({"e4m3": 4, "e5m2": 3, "nvf4": 2}[fmt])]
    assert len(pairs) > 300
    top = np.float32(2688.0 if fmt == "nvf4" else ref.TOP[fmt])
    rows = []
    for s24, x24 in pairs:
        s = np.float32(np.ldexp(float(s24), -23))
        most = np.float32(np.float64(top) * s)
        fits = [m for m in (most, np.nextafter(most, np.float32(0)), np.nextafter(most, np.float32(np.inf))) if m / top == s]
        if not fits:
            continue                        # no row has this scale
        row = np.zeros(64, np.float32)
        row[0] = fits[0]
        for k in range(32):
            row[32 + k] = np.ldexp(float(x24), -23 + (6 if fmt == "nvf4" else 8) - k) * (-1) ** k
        if fmt == "nvf4":                   # blocks of their own scale, largest first
            row[16:32] = row[32:48]
        rows.append(np.where(np.abs(row) <= row[0], row, 0))
    assert len(rows) > 100
    same(np.stack(rows), fmt)
