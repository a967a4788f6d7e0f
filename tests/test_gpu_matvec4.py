"""mmasim.matvec4 against its definition in 64 bits, and the operators together as a network would call them."""
import numpy as np
import pytest
import torch

import rows_ref as ref

pytestmark = pytest.mark.gpu
if torch.cuda.is_available():
    from paper_2511_10909_b200 import mmasim


def layer(N, K, fmt, seed=0):
    g = np.random.default_rng(seed + N + K)
    w = g.standard_normal((N, K), dtype=np.float32) / np.sqrt(K, dtype=np.float32)
    codes, sf, rs = ref.quantize(w, fmt)
    return codes, sf, rs


def cuda(a):
    return None if a is None else torch.from_numpy(np.ascontiguousarray(a)).cuda()


def tokens(T, K, dtype, seed=1):
    g = torch.Generator().manual_seed(seed + T + K)
    x = torch.randn((T, K), generator=g)
    x[:, :: max(1, K // 3)] *= 50
    return x.to(ref.DTYPES[dtype])


def check(y, x, codes, sf, rs, fmt, dtype):
    K = x.shape[1]
    x64, w64 = x.double().cpu().numpy(), ref.weights(codes, sf, fmt, rs)
    want = x64 @ w64.T
    bound = ref.matvec_bound(x64, w64, K)
    got = y.double().cpu().numpy()
    least = {"fp32": 2.0 ** -149, "bf16": 2.0 ** -133, "fp16": 2.0 ** -24}[dtype]
    most = torch.finfo(x.dtype).max
    with np.errstate(invalid="ignore"):
        near = np.abs(got - want) <= bound + ref.HALF_STEP[dtype] * (np.abs(want) + bound) + least
    over = (np.abs(want) + bound > most) & (got == np.sign(want) * np.inf)          # what passes the type is infinite,
    over |= (np.abs(x64) @ np.abs(w64).T > torch.finfo(torch.float32).max) & ~np.isfinite(got)      # what partial sums pass FP32 in, infinite or NaN
    assert y.dtype == x.dtype and (near | over).all(), np.argwhere(~(near | over))[:4].tolist()


@pytest.mark.parametrize("dtype", list(ref.DTYPES))
@pytest.mark.parametrize("fmt", ["mxf4", "nvf4"])
def test_matvec4(fmt, dtype):
    for T, N, K in [(1, 1, 32), (1, 17, 64), (2, 16, 96), (3, 100, 128), (1, 64, 160), (5, 33, 1024), (8, 48, 2080), (9, 20, 512), (1, 1111, 4128), (4, 272, 4096),
                    (16, 40, 8192), (2, 31, 16416), (17, 130, 288), (1, 2500, 512), (33, 64, 256), (7, 5000, 1024)]:
        codes, sf, rs = layer(N, K, fmt)
        x = tokens(T, K, dtype)
        check(mmasim.matvec4(fmt, cuda(ref.pack(codes, fmt)), cuda(sf), x.cuda(), cuda(rs)), x, codes, sf, rs, fmt, dtype)


@pytest.mark.parametrize("dtype", list(ref.DTYPES))
@pytest.mark.parametrize("fmt", ["mxf4", "nvf4"])
def test_whole_numbers_are_exact(fmt, dtype):
    """Every code and every token's own place: sums of small whole numbers (halves of them) have one value in FP32."""
    g = np.random.default_rng(2)
    for T, N, K in [(8, 40, 256), (3, 17, 2048), (1, 300, 96)]:
        codes = g.integers(0, 16, (N, K)).astype(np.uint8)
        sf = (np.exp2(g.integers(-2, 3, (N, K // ref.BLOCK[fmt]))))
        sf_codes = (np.log2(sf) + 127).astype(np.uint8) if fmt == "mxf4" else ((np.log2(sf) + 7).astype(np.uint8) << 3)
        x = torch.from_numpy(g.integers(-3, 4, (T, K)).astype(np.float32)).to(ref.DTYPES[dtype])
        y = mmasim.matvec4(fmt, cuda(ref.pack(codes, fmt)), cuda(sf_codes), x.cuda())
        want = x.double().numpy() @ ref.weights(codes, sf_codes, fmt).T
        assert np.array_equal(y.double().cpu().numpy(), torch.from_numpy(want).to(x.dtype).double().numpy())


def test_every_scale_code():
    """One row per scale byte; NaN scales, scales whose weights pass FP32, the smallest ones."""
    for fmt, K in (("mxf4", 64), ("nvf4", 32)):
        n = 256 if fmt == "mxf4" else 128
        codes = np.tile((np.arange(K) % 16).astype(np.uint8), (n, 1))
        sf = np.tile(np.arange(n, dtype=np.uint8)[:, None], (1, K // ref.BLOCK[fmt]))
        x = np.zeros((3, K), np.float32)
        x[0, 1], x[1, 7], x[2, 15] = 1.0, 2.0 ** -100, -3.0
        y = mmasim.matvec4(fmt, cuda(ref.pack(codes, fmt)), cuda(sf), cuda(x)).cpu().numpy()
        with np.errstate(all="ignore"):
            w = ref.weights(codes, sf, fmt)
            want = np.stack([w[:, 1] * 1.0, w[:, 7] * 2.0 ** -100, w[:, 15] * -3.0]).astype(np.float32)
            want[:, np.isnan(w).any(1)] = np.nan                                          # a NaN times the zeros of x
        # a product below 2^-126 has fewer bits
        least = 2.0 ** -149 * 256
        with np.errstate(invalid="ignore"):
            near = (y == want) | (np.abs(y - want) <= least) | (np.isnan(y) & np.isnan(want))     # (equal: infinities)
        assert near.all(), np.argwhere(~near)[:4].tolist()


def test_special_tokens():
    """An infinity or NaN in a token reaches that token's outputs alone."""
    codes, sf, rs = layer(40, 128, "nvf4")
    codes[:, 5] = np.where(np.arange(40) % 2, 2, 10)                      # +-1 under the infinity
    for dtype in ref.DTYPES:
        x = tokens(4, 128, dtype)
        x[1, 5] = float("inf")
        x[2, 9] = float("nan")
        y = mmasim.matvec4("nvf4", cuda(ref.pack(codes, "nvf4")), cuda(sf), x.cuda(), cuda(rs))
        assert torch.isfinite(y[0]).all() and torch.isfinite(y[3]).all() and torch.isnan(y[2]).all()
        assert (y[1] == torch.tensor([-float("inf"), float("inf")]).repeat(20).cuda().to(y.dtype)).all()
        check(y[[0, 3]], x[[0, 3]], codes, sf, rs, "nvf4", dtype)
    big = torch.tensor([[3.0e38, -3.0e38] + [0.0] * 30]).cuda()           # parts of the largest numbers
    codes = np.full((1, 32), 1, np.uint8)
    y = mmasim.matvec4("mxf4", cuda(ref.pack(codes, "mxf4")), cuda(np.full((1, 1), 127, np.uint8)), big)
    assert y.item() == 0.0


@pytest.mark.parametrize("dtype", list(ref.DTYPES))
@pytest.mark.parametrize("fmt", ["mxf4", "nvf4"])
def test_far_apart_magnitudes(fmt, dtype):
    """Tokens whose elements lie further apart than 16 bits hold (some of them where every weight is zero), blocks whose scales do."""
    g = np.random.default_rng(3)
    for T, N, K in [(1, 40, 256), (3, 33, 1056), (9, 100, 544)]:
        codes = g.integers(0, 16, (N, K)).astype(np.uint8)
        sf = (g.integers(60, 200, (N, K // 32)) if fmt == "mxf4" else g.integers(0, 127, (N, K // 16))).astype(np.uint8)
        if fmt == "mxf4":
            sf[::3] = g.integers(100, 140, sf[::3].shape)               # some rows near together, one of them with zero blocks under far scales
            sf[1::3] = 127
            sf[1, ::2] = 3
            codes[1, (np.arange(K) // 32) % 2 == 0] &= 8
            sf[4, -1] = 251
        x = g.standard_normal((T, K)) * np.exp2(g.integers(-12, 6, (T, K)))
        big = np.array([5, 130, K - 3])
        codes[:, big] &= 8                                               # zeros of both signs
        if dtype != "fp16":
            x *= np.where(g.random((T, K)) < 0.02, 2.0 ** -45, 1.0)
            x[:, 5], x[:, 130] = 3e38, -1e25
        x[:, K - 3] = 6e4
        x = torch.from_numpy(x).to(ref.DTYPES[dtype])
        check(mmasim.matvec4(fmt, cuda(ref.pack(codes, fmt)), cuda(sf), x.cuda()), x, codes, sf, None, fmt, dtype)


def test_strides_outputs_and_streams():
    N, K, T = 50, 352, 3
    for fmt in ("mxf4", "nvf4"):
        codes, sf, rs = layer(N, K, fmt)
        W, sf, rs = cuda(ref.pack(codes, fmt)), cuda(sf), cuda(rs)
        for dtype in ref.DTYPES:
            x = tokens(T, K, dtype).cuda()
            want = mmasim.matvec4(fmt, W, sf, x, rs)
            wide = torch.zeros((N, K // 2 + 48), dtype=torch.uint8, device="cuda")
            wide[:, :K // 2] = W
            for off in (0, 1, 8):
                xb = torch.full((T, K + 24), float("nan"), dtype=x.dtype, device="cuda")
                xb[:, off:off + K] = x
                out = torch.full((T, N + 7), 7.0, dtype=x.dtype, device="cuda")
                y = mmasim.matvec4(fmt, wide[:, :K // 2], sf, xb[:, off:off + K], rs, out=out[:, 2:2 + N])
                assert torch.equal(y, want) and (out[:, :2] == 7).all() and (out[:, 2 + N:] == 7).all()
            side = torch.cuda.Stream()
            side.wait_stream(torch.cuda.current_stream())
            y = mmasim.matvec4(fmt, W, sf, x, rs, stream=side)
            side.synchronize()
            assert torch.equal(y, want)
            sx = torch.zeros_like(x)
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph):
                y = mmasim.matvec4(fmt, W, sf, sx, rs)
            sx.copy_(x)
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(y, want)
    assert mmasim.matvec4("mxf4", W, sf[:, ::2].contiguous(), x[:0]).shape == (0, N)


@pytest.mark.parametrize("dtype,K", [("fp32", 20480), ("fp32", 20448), ("bf16", 32768), ("fp16", 32736)])
@pytest.mark.parametrize("fmt", ["mxf4", "nvf4"])
def test_longest_rows(fmt, dtype, K):
    """Shared memory then holds few tokens: calls for several read the weights more than once."""
    codes, sf, rs = layer(40, K, fmt)
    for T in (1, 2, 3, 7):
        x = tokens(T, K, dtype)
        check(mmasim.matvec4(fmt, cuda(ref.pack(codes, fmt)), cuda(sf), x.cuda(), cuda(rs)), x, codes, sf, rs, fmt, dtype)


def test_weights_beyond_32_bits():
    """Rows of a matrix whose offsets pass 2^32 bytes."""
    K, N, ld = 64, 3, (1 << 31) + 32                                       # bytes between rows
    buf = torch.zeros((2 * ld + K,), dtype=torch.uint8, device="cuda")
    W = torch.as_strided(buf, (N, K // 2), (ld, 1))
    codes, sf, _ = layer(N, K, "mxf4")
    W.copy_(cuda(ref.pack(codes, "mxf4")))
    x = tokens(2, K, "bf16")
    check(mmasim.matvec4("mxf4", W, cuda(sf), x.cuda()), x, codes, sf, None, "mxf4", "bf16")


def test_refusals():
    codes, sf, rs = layer(16, 64, "nvf4")
    W, sf, rs = cuda(ref.pack(codes, "nvf4")), cuda(sf), cuda(rs)
    x = torch.randn((2, 64), device="cuda")

    def refused(status, *a, **kw):
        with pytest.raises(mmasim.MmasimError) as e:
            mmasim.matvec4(*a, **kw)
        assert e.value.status == status, e.value

    refused(2, "e4m3", W, sf, x, rs)
    refused(1, "nvf4", W, sf, x.cpu(), rs)
    refused(1, "nvf4", W, sf, x.double(), rs)
    refused(3, "nvf4", W, sf, x[:, :48], rs)
    refused(3, "nvf4", W[:, :16], sf, x, rs)
    refused(3, "nvf4", W, sf[:, :2], x, rs)
    refused(3, "mxf4", W, sf, x)
    refused(3, "nvf4", W, sf, x, rs[:8])
    refused(1, "nvf4", W, sf, x, rs, out=torch.empty((2, 16), dtype=torch.float16, device="cuda"))
    wide = torch.zeros((16, 40), dtype=torch.uint8, device="cuda")
    refused(4, "nvf4", wide[:, :32], sf, x, rs)                            # rows that do not start on 16 bytes
    refused(4, "nvf4", torch.zeros(16 * 32 + 8, dtype=torch.uint8, device="cuda")[8:].view(16, 32), sf, x, rs)
    sq = torch.randn((2, 64), device="cuda")
    codes, s4, r4 = layer(64, 64, "nvf4")
    refused(1, "nvf4", cuda(ref.pack(codes, "nvf4")), cuda(s4), sq, cuda(r4), out=sq)


def test_operators_together():
    """A block of a network that generates, on the operators and the products of the library: h = x + residual, its norm into NVFP4, the
    product of both 4-bit operands under Blackwell's arithmetic, and the weight-only product of the same weights from the plain norm."""
    g = torch.Generator().manual_seed(11)
    T, K, N = 4, 512, 384
    x, res = (torch.randn((T, K), generator=g).to(torch.bfloat16).cuda() for _ in range(2))
    gain = (1 + 0.1 * torch.randn(K, generator=g)).cuda()
    wt = (torch.randn((N, K), generator=g) / K ** 0.5).to(torch.bfloat16).cuda()
    w = mmasim.quantize(wt, "nvf4")
    q, h = mmasim.rms_norm(x, gain, res, fmt="nvf4")
    y, h2 = mmasim.rms_norm(x, gain, res)
    assert torch.equal(h, h2)
    model = mmasim.Model("blackwell", "nvf4", "fp32")
    D = mmasim.gemm(model, q.codes, w.codes, sfa=q.sf, sfb=w.sf, row_scale=q.row_scale, col_scale=w.row_scale).view(torch.float32)
    host = lambda m: tuple(None if t is None else t.cpu().numpy() for t in m)
    (qc, qs, qr), (wc, ws, wr) = host(q), host(w)
    w64 = ref.weights(ref.unpack(wc, "nvf4"), ws, "nvf4", wr)
    q64 = ref.weights(ref.unpack(qc, "nvf4"), qs, "nvf4", qr)
    # the model: F = 35 bits of groups, RZ-FP32 per 64 elements, two scales: a few units of FP32 per block
    assert (np.abs(D.double().cpu().numpy() - q64 @ w64.T) <= (2 * K // 64 + 6) * 2.0 ** -23 * (np.abs(q64) @ np.abs(w64).T)).all()
    direct = mmasim.matvec4("nvf4", w.codes, w.sf, y, w.row_scale)
    check(direct, y, ref.unpack(wc, "nvf4"), ws, wr, "nvf4", "bf16")
    # FP8 rows through the Hopper model, with row scales on both sides
    w8 = mmasim.quantize(wt, "e4m3")
    q8, _ = mmasim.rms_norm(x, gain, res, fmt="e4m3")
    D8 = mmasim.gemm(mmasim.Model("blackwell", "e4m3", "fp32"), q8.codes, w8.codes, row_scale=q8.row_scale, col_scale=w8.row_scale).view(torch.float32)
    a64, b64 = (t.codes.view(torch.float8_e4m3fn).double() * t.row_scale.double()[:, None] for t in (q8, w8))
    assert ((D8.double() - a64 @ b64.T).abs() <= (33 * K // 32 + 6) * 2.0 ** -23 * (a64.abs() @ b64.abs().T)).all()
    # MX operands, and the backward pass of the block through the weight-only weights
    qm, _ = mmasim.rms_norm(x, gain, res, fmt="mxe4m3")
    wm = mmasim.quantize(wt, "mxe4m3")
    Dm = mmasim.gemm(mmasim.Model("blackwell", "mxe4m3", "fp32"), qm.codes, wm.codes, sfa=qm.sf, sfb=wm.sf).view(torch.float32)
    a64, b64 = (torch.from_numpy(ref.code_values(t.codes.cpu().numpy(), "mxe4m3") * ref.units((None, t.sf.cpu().numpy(), None), "mxe4m3", K)) for t in (qm, wm))
    assert ((Dm.double().cpu() - a64 @ b64.T).abs() <= (33 * K // 32 + 6) * 2.0 ** -23 * (a64.abs() @ b64.abs().T)).all()
    dy = (torch.randn((T, N), generator=g).cuda().double() @ torch.from_numpy(w64).cuda()).to(torch.bfloat16)
    dx, dgain = mmasim.rms_norm_backward(dy, h, gain, res)
    n64 = lambda t: t.double().cpu().numpy()
    dx64, dw64, bx, bw = ref.rms_norm_backward(n64(dy), n64(h), n64(gain), n64(res), float(np.float32(1e-6)))
    assert (np.abs(n64(dx) - dx64) <= bx + ref.HALF_STEP["bf16"] * (np.abs(dx64) + bx)).all()
    assert (np.abs(n64(dgain) - dw64) <= bw + ref.U * (np.abs(dw64) + bw)).all()
