"""mmasim.matvec4 of tokens near their type's lower end, beside ordinary elements and alone: products stay exact."""
import numpy as np
import pytest
import torch

import rows_ref as ref

pytestmark = pytest.mark.gpu
if torch.cuda.is_available():
    from paper_2511_10909_b200 import mmasim


def check(fmt, x, codes, sf, rs, half=ref.U, least=2.0 ** -149):
    K = x.shape[1]
    cuda = lambda a: None if a is None else torch.from_numpy(np.ascontiguousarray(a)).cuda()
    y = mmasim.matvec4(fmt, cuda(ref.pack(codes, fmt)), cuda(sf), x.cuda() if torch.is_tensor(x) else cuda(x), cuda(rs)).double().cpu().numpy()
    x64, w64 = x.double().numpy() if torch.is_tensor(x) else x.astype(np.float64), ref.weights(codes, sf, fmt, rs)
    want = x64 @ w64.T
    # as in matvec_bound; a sum below 2^-126 is off by up to 2^-150 at every addition, of which there are at most K + 16, before the row's scale (< 2)
    bound = ref.matvec_bound(x64, w64, K) + (K + 16) * 2.0 ** -149
    bad = ~(np.abs(y - want) <= bound + half * (np.abs(want) + bound) + least)
    assert not bad.any(), [(y[tuple(i)], want[tuple(i)]) for i in np.argwhere(bad)[:3]]


@pytest.mark.parametrize("power", [-60, -100, -112, -120, -126, -132, -140, -146])
@pytest.mark.parametrize("fmt", ["mxf4", "nvf4"])
def test_small_tokens(fmt, power):
    """Whole tokens of that size, and some elements of that size among ordinary ones that meet weights of zero."""
    for T, N, K in [(1, 40, 96), (3, 33, 512), (5, 17, 1056), (2, 50, 256), (7, 20, 288)]:
        g = np.random.default_rng(T + N + K)
        codes = g.integers(0, 16, (N, K)).astype(np.uint8)
        sf = (g.integers(120, 160, (N, K // 32)) if fmt == "mxf4" else g.integers(1, 127, (N, K // 16))).astype(np.uint8)
        rs = g.random(N).astype(np.float32) + 0.5 if fmt == "nvf4" else None
        x = (g.standard_normal((T, K)) * 2.0 ** power * np.exp2(g.integers(-8, 9, (T, K)))).astype(np.float32)
        x[0, 0] = np.float32(2.0 ** power)
        check(fmt, x, codes, sf, rs)
        x[:, 1::3] = g.standard_normal(x[:, 1::3].shape).astype(np.float32)
        codes[:, 1::3] &= 8                 # zeros of both signs
        check(fmt, x, codes, sf, rs)


@pytest.mark.parametrize("power", [-60, -95, -100, -110, -120, -126])
@pytest.mark.parametrize("fmt", ["mxf4", "nvf4"])
def test_small_bf16_tokens(fmt, power):
    """Outputs far above BF16's smallest numbers (scales of 2^20 and more), so that what is lost on the way would show."""
    for T, N, K in [(1, 40, 96), (3, 33, 512), (9, 17, 1056), (2, 50, 256)]:
        g = np.random.default_rng(T + N + K)
        codes = g.integers(0, 16, (N, K)).astype(np.uint8)
        sf = (g.integers(150, 170, (N, K // 32)) if fmt == "mxf4" else g.integers(1, 127, (N, K // 16))).astype(np.uint8)
        x = torch.from_numpy(g.standard_normal((T, K)) * 2.0 ** power * np.exp2(g.integers(-3, 4, (T, K)))).to(torch.bfloat16)
        check(fmt, x, codes, sf, None, ref.HALF_STEP["bf16"], 2.0 ** -134)
        x[:, 1::3] = 1.0
        codes[:, 1::3] &= 8                 # zeros of both signs
        check(fmt, x, codes, sf, None, ref.HALF_STEP["bf16"], 2.0 ** -134)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_weights_beyond_fp32_in_the_last_block(dtype):
    """One weight of 6 x 2^127 under an x of 1: infinite, also where lanes behind the last block of a step that FP16 does not hold repeat its weights."""
    for T in (1, 2, 4, 9):
        for K in (32, 96, 288, 320):
            codes = np.zeros((18, K), np.uint8)
            sf = np.full((18, K // 32), 127, np.uint8)
            codes[:, K - 5], sf[:, -1] = np.where(np.arange(18) % 2, 7, 15), 254
            x = torch.ones((T, K))
            x[:, K - 9], x[:, K - 7] = 1e25, 2.0 ** -45
            y = mmasim.matvec4("mxf4", torch.from_numpy(ref.pack(codes, "mxf4")).cuda(), torch.from_numpy(sf).cuda(), x.to(ref.DTYPES[dtype]).cuda()).cpu().float()
            assert torch.equal(y, torch.tensor([-float("inf"), float("inf")]).repeat(T, 9)), (T, K)
