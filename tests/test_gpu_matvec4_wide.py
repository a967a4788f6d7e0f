"""mmasim.matvec4 of many outputs, where 2 or 4 warps share a tile of 16 rows and rounds of other splits follow."""
import numpy as np
import pytest
import torch

import rows_ref as ref

pytestmark = pytest.mark.gpu
if torch.cuda.is_available():
    from paper_2511_10909_b200 import mmasim

# outputs -> how many warps share a tile, round by round (148 CTAs, tiles of 16 rows)
ROUNDS = {7200: (4,), 14337: (4, 8, 16), 16600: (2,), 28667: (2, 4, 16), 21001: (2, 16), 46000: (2, 2, 4)}


def splits(N, ctas=148):
    """Rounds by the rule of the kernel: as few warps a tile as still have a tile each."""
    left, rounds = -(-N // 16), []
    while left > 0:
        split = 2 if left > 7 * ctas else 4 if left > 3 * ctas else 8 if left > ctas else 16
        rounds.append(split)
        left -= 16 // split * ctas
    return tuple(rounds)


def layer(N, K, fmt, seed):
    g = np.random.default_rng(seed + N + K)
    codes = g.integers(0, 16, (N, K)).astype(np.uint8)
    sf = (g.integers(117, 131, (N, K // 32)) if fmt == "mxf4" else g.integers(8, 90, (N, K // 16))).astype(np.uint8)
    return codes, sf, (g.random(N).astype(np.float32) + 0.5 if fmt == "nvf4" else None)


def check(fmt, dtype, T, N, K, seed, far=False):
    codes, sf, rs = layer(N, K, fmt, seed)
    g = torch.Generator().manual_seed(seed + T)
    x = torch.randn((T, K), generator=g)
    if far:                                 # elements that FP16 parts do not hold beside one another, in one step of 256, the large one times zeros
        x[T - 1, K // 2], x[T - 1, K // 2 + 1] = 1e25, 2.0 ** -45
        codes[:, K // 2] &= 8
    x = x.to(ref.DTYPES[dtype])
    cuda = lambda a: None if a is None else torch.from_numpy(np.ascontiguousarray(a)).cuda()
    y = mmasim.matvec4(fmt, cuda(ref.pack(codes, fmt)), cuda(sf), x.cuda(), cuda(rs))
    x64, w64 = x.double().numpy(), ref.weights(codes, sf, fmt, rs)
    want = x64 @ w64.T
    # 128 products by eight instructions that truncate 17 terms 2^-24 below the largest; two sums a step of 256, the steps shared by two warps
    # at the fewest; the two halves of a sum, the lanes of a token, at most eight warps' pairs, three parts, the row's scale
    bound = (8 * 18 + 2 * -(-K // 512) + 16) * ref.U * (np.abs(x64) @ np.abs(w64).T)
    least = {"fp32": 2.0 ** -149, "bf16": 2.0 ** -133, "fp16": 2.0 ** -24}[dtype]
    err = np.abs(y.double().cpu().numpy() - want)
    bad = ~(err <= bound + ref.HALF_STEP[dtype] * (np.abs(want) + bound) + least)
    if dtype == "fp16":
        bad &= np.abs(want) + bound <= torch.finfo(torch.float16).max
    assert not bad.any(), np.argwhere(bad)[:4].tolist()


def test_the_sizes_reach_every_split():
    assert {N: splits(N) for N in ROUNDS} == ROUNDS


@pytest.mark.parametrize("N", list(ROUNDS))
@pytest.mark.parametrize("fmt", ["mxf4", "nvf4"])
def test_many_outputs(fmt, N):
    for i, (dtype, T, K) in enumerate([("bf16", 1, 96), ("fp16", 3, 512), ("fp32", 1, 352), ("bf16", 9, 800), ("fp16", 2, 1312), ("fp32", 3, 256), ("bf16", 16, 1024), ("fp32", 5, 608)]):
        check(fmt, dtype, T, N, K, i)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("fmt", ["mxf4", "nvf4"])
def test_steps_that_are_not_exact(fmt, dtype):
    for T, N, K in [(1, 28667, 640), (3, 16600, 768), (4, 14337, 544)]:
        check(fmt, dtype, T, N, K, 11, far=True)


def test_long_rows_of_two_warps():
    check("nvf4", "bf16", 1, 16600, 8192, 5)
    check("mxf4", "fp16", 4, 16600, 4128, 6)
