"""mmasim.rms_norm and rms_norm_backward of rows far from one: magnitudes whose squares are still FP32 numbers, and those whose are not."""
import numpy as np
import pytest
import torch

import rows_ref as ref

pytestmark = pytest.mark.gpu
if torch.cuda.is_available():
    from paper_2511_10909_b200 import mmasim

# the ring of copies (16-byte accesses), rows of a few threads, elements spread over the threads, rows read twice (FP32, 16385 and more)
SIZES = [(5, 256), (700, 64), (3, 4096), (4, 257), (650, 1111), (3, 40), (2, 32768)]


def np64(t):
    return t.detach().cpu().double().numpy()


def rows(M, K, dtype, mag, seed):
    """h of magnitude `mag` (a power of two of its own for every row, -3 .. 3), and a gradient that lies along it for the most part: there the
    two terms of dx are of one size."""
    g = torch.Generator().manual_seed(seed + M + K)
    unit = torch.randn((M, K), generator=g)
    h = (unit.double() * torch.exp2(torch.randint(-3, 4, (M, 1), generator=g).double()) * mag).to(ref.DTYPES[dtype])
    dy = ((0.9 * unit + 0.3 * torch.randn((M, K), generator=g)) * torch.exp2(torch.randint(-3, 4, (M, 1), generator=g).float())).to(ref.DTYPES[dtype])
    return h, dy


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("mag,eps", [(1e12, 1e-6), (1e14, 1e-6), (1e15, 1e-6), (1e16, 0.0), (1e-13, 0.0), (1e-15, 0.0), (1e-16, 0.0)])
def test_gradients_of_far_rows(mag, eps, dtype):
    """dx where r^3 leaves FP32 and dx does not.

    Bounds of rows_ref.rms_norm_backward.  They hold for dx = r (g - (h r) m) with m = (r sum(g h)) / K: r is known to 43 U; the term r g has 46
    (the product with the weight, the subtraction, r and its product; 48 allowed); h r 44, m 43 + 3 and the sum's own 74 of its terms'
    magnitudes, their subtraction, r and its product 45: 135 of the second term (140 allowed) and 74 of the magnitudes (78); the residual is
    added with dx's own rounding."""
    for i, (M, K) in enumerate(SIZES):
        h, dy = rows(M, K, dtype, mag, i)
        w = None if i % 3 == 0 else 1 + 0.2 * torch.randn(K, generator=torch.Generator().manual_seed(K))
        if i % 3 == 1:
            w = w.to(h.dtype)
        res = None if i % 2 else (torch.randn((M, K), generator=torch.Generator().manual_seed(7)).double() / mag).to(h.dtype)
        cuda = lambda t: None if t is None else t.cuda()
        dx, dw = mmasim.rms_norm_backward(dy.cuda(), h.cuda(), cuda(w), cuda(res), eps=eps)
        dx64, dw64, dx_bound, dw_bound = ref.rms_norm_backward(np64(dy), np64(h), None if w is None else np64(w), None if res is None else np64(res), float(np.float32(eps)))
        half, least = ref.HALF_STEP[dtype], {"fp32": 2.0 ** -149, "bf16": 2.0 ** -133}[dtype]
        err = np.abs(np64(dx) - dx64)
        assert (err <= dx_bound + half * (np.abs(dx64) + dx_bound) + least).all(), (M, K, (err / np.abs(dx64).max(1, keepdims=True)).max())
        wh = half if w is None or w.dtype != torch.float32 else ref.HALF_STEP["fp32"]
        err = np.abs(np64(dw) - dw64)
        assert (err <= dw_bound + wh * (np.abs(dw64) + dw_bound) + least).all(), (M, K, err.max())


@pytest.mark.parametrize("K", [256, 257])
def test_small_gradients_of_large_rows(K):
    """Row times r before anything else: r^2 alone, times a gradient of 2^-17, would be subnormal here."""
    h, dy = rows(6, K, "fp32", 1e16, 3)
    dy *= 2.0 ** -17
    dx, _ = mmasim.rms_norm_backward(dy.cuda(), (h * 8).cuda())
    dx64, _, bound, _ = ref.rms_norm_backward(np64(dy), np64(h * 8), None, None, 1e-6)
    assert (np.abs(np64(dx) - dx64) <= bound + ref.U * (np.abs(dx64) + bound)).all()


def test_where_the_squares_leave_fp32():
    """A row of 4096 elements passes FP32's range of squares at magnitudes of 2.9e17, far below one element's 1.8e19."""
    K = 4096
    sign = torch.where(torch.rand((4, K), generator=torch.Generator().manual_seed(1)) < 0.5, -1.0, 1.0)
    h = (sign * torch.tensor([[1e17], [2.8e17], [3.0e17], [1e19]])).cuda()
    y, _ = mmasim.rms_norm(h)
    assert (y[2:] == 0).all() and (y[:2].cpu() - sign[:2]).abs().max() <= 2 * ref.NORM_REL
    dy, res = torch.randn((4, K), generator=torch.Generator().manual_seed(2)).cuda(), torch.randn((4, K), generator=torch.Generator().manual_seed(3)).cuda()
    dx, dw = mmasim.rms_norm_backward(dy, h, None, res)
    assert torch.equal(dx[2:], res[2:])
    assert torch.equal(dw, mmasim.rms_norm_backward(dy[:2], h[:2])[1])
    assert (mmasim.rms_norm_backward(dy, h)[0][2:] == 0).all()


def test_small_rows_without_eps():
    """Down to mean squares of 2^-126 a row's norm is as good as any; where the squares vanish there is nothing to divide by."""
    x = torch.randn((3, 500), generator=torch.Generator().manual_seed(5))
    for mag in (1e-12, 1e-16, 1e-18):
        h = x * mag
        y, _ = mmasim.rms_norm(h.cuda(), eps=0.0)
        y64, _ = ref.rms_norm(np64(h), None, 0.0)
        # squares below 2^-126 are off by up to 2^-150 each
        assert (np.abs(np64(y) - y64) <= np.abs(y64) * (ref.NORM_REL + ref.U + 2.0 ** -150 / (np64(h) ** 2).mean(1, keepdims=True))).all(), mag
    h = torch.tensor([[1e-24, -1e-25, 0.0, 1e-30]]).cuda()
    assert torch.isnan(mmasim.rms_norm(h, eps=0.0)[0]).all()
