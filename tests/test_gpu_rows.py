"""mmasim.quantize, rms_norm and rms_norm_backward against their definitions (rows_ref)."""
import numpy as np
import pytest
import torch

import rows_ref as ref

pytestmark = pytest.mark.gpu
if torch.cuda.is_available():
    from paper_2511_10909_b200 import mmasim

SIZES = [(1, 1), (1, 7), (3, 8), (5, 31), (2, 32), (1, 33), (7, 64), (9, 100), (33, 128), (5, 250), (4, 257), (3, 1000), (2, 1111), (3, 4096), (2, 4100),
         (2, 8192), (1, 16392), (2, 32768)]


def rows(M, K, dtype, seed=0, scale=1.0):
    g = torch.Generator().manual_seed(seed + 1000 * M + K)
    x = torch.randn((M, K), generator=g) * torch.exp2(torch.randint(-6, 7, (M, 1), generator=g).float()) * scale
    x[torch.rand((M, K), generator=g) < 0.02] *= 30
    return x.to(ref.DTYPES[dtype])


def np64(t):
    return t.detach().cpu().double().numpy()


def host(q, fmt):
    c, sf, s = (None if t is None else t.cpu().numpy() for t in q)
    return ref.unpack(c, fmt), sf, s


def assert_same(q, want, fmt):
    for name, a, b in zip(("codes", "sf", "row_scale"), host(q, fmt), want):
        assert (a is None) == (b is None), name
        if a is not None:
            assert a.shape == b.shape, name
            bad = np.argwhere(a.view(np.uint32 if a.dtype == np.float32 else np.uint8) != b.view(np.uint32 if b.dtype == np.float32 else np.uint8)) \
                if name != "row_scale" else np.argwhere(~((a == b) | (np.isnan(a) & np.isnan(b))))
            assert bad.size == 0, (name, len(bad), bad[0], a[tuple(bad[0])], b[tuple(bad[0])])


@pytest.mark.parametrize("dtype", list(ref.DTYPES))
@pytest.mark.parametrize("fmt", ref.FORMATS)
def test_quantize_is_its_definition(fmt, dtype):
    for M, K in SIZES:
        if fmt in ("mxf4", "nvf4"):
            K = -(-K // 32) * 32
        x = rows(M, K, dtype)
        assert_same(mmasim.quantize(x.cuda(), fmt), ref.quantize(x.float().numpy(), fmt), fmt)


@pytest.mark.parametrize("fmt", ref.FORMATS)
def test_quantize_extremes(fmt):
    """Zeros, subnormals, the largest numbers, ties, one outlier, infinities and NaN."""
    g = torch.Generator().manual_seed(5)
    K = 96
    x = torch.randn((24, K), generator=g)
    x[0] = 0
    x[1] = -0.0
    x[2] *= 2.0 ** -140
    x[3] *= 2.0 ** -120
    x[4] *= 2.0 ** -100
    x[5] *= 2.0 ** -80
    x[6] = x[6].clamp(-1, 1) * 3.0e38
    x[7, 40] = 3.4028234663852886e38
    x[8, 3] = 1e30
    x[9, 5] = float("inf")
    x[10, 70] = -float("inf")
    x[11, 95] = float("nan")
    x[12] = torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.0] * 12)
    x[13] = torch.tensor([-0.25, 0.5, -1.5, 2.25, -2.75, 3.25, 4.5, -6.0] * 12)
    x[14] = torch.arange(K) * 2.0 ** -9 * 448 / 96
    x[15] = torch.where(torch.arange(K) < 32, 0.0, x[15])
    x[16] = 2.0 ** torch.arange(-60, 36).float()
    x[17] = 2.0 ** torch.arange(-149, -53).float()
    x[18] = 448.0 * 2.0 ** -126
    x[19] = torch.nextafter(torch.tensor(2.0 ** -60 * 448), torch.tensor(1.0))
    x[20] = 2.0 ** -60 * 448 * torch.rand(K, generator=g)
    x[21] = 1.0 - 2.0 ** -24
    assert_same(mmasim.quantize(x.cuda(), fmt), ref.quantize(x.numpy(), fmt), fmt)


@pytest.mark.parametrize("dtype", list(ref.DTYPES))
@pytest.mark.parametrize("fmt", ref.FORMATS)
def test_zeros_keep_their_signs(fmt, dtype):
    for M, K in [(40, 96), (3, 4096), (7, 1000 if fmt not in ("mxf4", "nvf4") else 992)]:
        x = rows(M, K, dtype, 2)
        x[:, ::5] = 0.0
        x[:, 1::7] = -0.0
        assert_same(mmasim.quantize(x.cuda(), fmt), ref.quantize(x.float().numpy(), fmt), fmt)


@pytest.mark.parametrize("fmt", ["e4m3", "e5m2", "nvf4"])
def test_quotients_are_rounded_as_division_rounds_them(fmt):
    """Rows around the codes' ties: quotients next to one differ in their last bits."""
    g = torch.Generator().manual_seed(8)
    tie = {"e4m3": 8, "e5m2": 4, "nvf4": 2}[fmt]
    M, K = 256, 4096
    s = torch.rand((M, 1), generator=g) + 0.5
    x = (torch.randint(0, 16 * tie, (M, K), generator=g) + 0.5) / tie * s
    x = torch.where(torch.rand((M, K), generator=g) < 0.3, torch.nextafter(x, torch.tensor(0.0)), x)
    x[:, 0] = ref.TOP[ref.elem(fmt)] * s[:, 0] if fmt != "nvf4" else 2688 * s[:, 0]
    assert_same(mmasim.quantize(x.cuda(), fmt), ref.quantize(x.numpy(), fmt), fmt)


def norm_case(M, K, dtype, residual, wide, seed=0):
    x, res = rows(M, K, dtype, seed), rows(M, K, dtype, seed + 1) if residual else None
    w = None
    if wide is not None:
        w = 1 + 0.2 * torch.randn(K, generator=torch.Generator().manual_seed(K))
        w = w if wide else w.to(x.dtype)
    h = x if res is None else (x.float() + res.float()).to(x.dtype)
    return x, res, w, h


def check_norm(y, h_got, x, res, w, h, dtype, fmt, eps):
    if res is None:
        assert h_got is None
    else:
        assert torch.equal(h_got.cpu(), h)
    y64, _ = ref.rms_norm(np64(h), None if w is None else np64(w), eps)
    if fmt is None:
        assert y.dtype == x.dtype
        half = ref.HALF_STEP[dtype]
        least = {"fp32": 2.0 ** -149, "bf16": 2.0 ** -133, "fp16": 2.0 ** -24}[dtype]
        assert (np.abs(np64(y) - y64) <= np.abs(y64) * (ref.NORM_REL + half * (1 + ref.NORM_REL)) + least).all()
    else:
        ref.assert_quantised(host(y, fmt), y64, fmt, ref.NORM_REL)


@pytest.mark.parametrize("dtype", list(ref.DTYPES))
@pytest.mark.parametrize("fmt", [None] + ref.FORMATS)
def test_rms_norm(fmt, dtype):
    for i, (M, K) in enumerate(SIZES):
        if fmt in ("mxf4", "nvf4"):
            K = -(-K // 32) * 32
        x, res, w, h = norm_case(M, K, dtype, i % 3 != 0, [None, False, True][(i // 2) % 3])
        y, h_got = mmasim.rms_norm(x.cuda(), None if w is None else w.cuda(), None if res is None else res.cuda(), eps=1e-5, fmt=fmt)
        check_norm(y, h_got, x, res, w, h, dtype, fmt, float(np.float32(1e-5)))


def test_rms_norm_of_special_rows():
    x = torch.randn((6, 40), generator=torch.Generator().manual_seed(3))
    x[0] = 0
    x[1, 7] = float("nan")
    x[2, 8] = float("inf")
    x[3] = 1e25                             # squares pass FP32: zeros
    x[4] *= 1e-30                           # eps is all there is
    y, _ = mmasim.rms_norm(x.cuda(), eps=1e-6)
    y = y.cpu()
    assert (y[0] == 0).all() and torch.isnan(y[1]).all()
    assert torch.isnan(y[2, 8]) and (y[2, :8] == 0).all() and (y[3] == 0).all()
    assert torch.allclose(y[4], x[4] * 1e3, rtol=1e-5, atol=0)
    for fmt in ref.FORMATS[:2]:
        q, _ = mmasim.rms_norm(x.cuda(), fmt=fmt)
        assert torch.isnan(q.row_scale.cpu()).tolist() == [False, True, True, False, False, False]
        assert (q.codes[1:3].cpu() == 0x7F).all()
    y, _ = mmasim.rms_norm(torch.zeros((2, 8), device="cuda"), eps=0.0)
    assert torch.isnan(y).all()             # 0 / 0


def check_backward(dx, dw, dy, x, w, res, dtype, eps):
    dx64, dw64, dx_bound, dw_bound = ref.rms_norm_backward(np64(dy), np64(x), None if w is None else np64(w), None if res is None else np64(res), eps)
    half, least = ref.HALF_STEP[dtype], {"fp32": 2.0 ** -149, "bf16": 2.0 ** -133, "fp16": 2.0 ** -24}[dtype]
    err = np.abs(np64(dx) - dx64)
    assert (err <= dx_bound + half * (np.abs(dx64) + dx_bound) + least).all(), (x.shape, err.max())
    wh = half if w is None or w.dtype != torch.float32 else ref.HALF_STEP["fp32"]
    assert dw.dtype == (x.dtype if w is None else w.dtype)
    err = np.abs(np64(dw) - dw64)
    assert (err <= dw_bound + wh * (np.abs(dw64) + dw_bound) + least).all(), (x.shape, err.max())


@pytest.mark.parametrize("dtype", list(ref.DTYPES))
def test_rms_norm_backward(dtype):
    for i, (M, K) in enumerate(SIZES + [(700, 64), (2000, 40), (300, 520), (650, 1111), (400, 2048)]):
        x, res, w, _ = norm_case(M, K, dtype, i % 2 == 0, [None, False, True][i % 3], seed=7)
        dy = rows(M, K, dtype, 9, 0.1)
        dx, dw = mmasim.rms_norm_backward(dy.cuda(), x.cuda(), None if w is None else w.cuda(), None if res is None else res.cuda(), eps=1e-5)
        check_backward(dx, dw, dy, x, w, res, dtype, float(np.float32(1e-5)))


def test_backward_is_the_gradient_of_the_forward_pass():
    """Central differences of the library's own FP32 norm, along random directions, against its gradients."""
    M, K, eps = 4, 96, 1e-3
    g = torch.Generator().manual_seed(4)
    x, w, dy, res = (torch.randn(s, generator=g).cuda() for s in ((M, K), (K,), (M, K), (M, K)))
    dh = torch.randn((M, K), generator=g).cuda()

    def loss(x, w):
        y, h = mmasim.rms_norm(x, w, res, eps=eps)
        return ((y.double() * dy.double()).sum() + (h.double() * dh.double()).sum()).item()

    dx, dw = mmasim.rms_norm_backward(dy, x + res, w, dh, eps=eps)
    step = 2.0 ** -7
    for k in range(4):
        dirx, dirw = (torch.randn(s, generator=g).cuda() for s in ((M, K), (K,)))
        for num, want in ((loss(x + step * dirx, w) - loss(x - step * dirx, w), (dx.double() * dirx).sum().item()),
                          (loss(x, w + step * dirw) - loss(x, w - step * dirw), (dw.double() * dirw).sum().item())):
            # FP32 outputs known to 2^-20, divided by the step: 2^-12 of the sums' magnitudes; third derivatives times step^2: 2^-14
            scale = (dy.abs().sum() + dh.abs().sum()).item()
            assert abs(num / (2 * step) - want) <= 2.0 ** -11 * scale


# ---- how the calls are made ----
def strided(t, lead, off):
    """A CUDA copy of t with `lead` more elements a row, starting `off` elements into its buffer; the rest is NaN."""
    M, K = t.shape
    buf = torch.full((M * (K + lead) + off + 8,), float("nan"), dtype=t.dtype, device="cuda")
    v = buf[off:off + M * (K + lead)].view(M, K + lead)[:, :K]
    v.copy_(t)
    return v


@pytest.mark.parametrize("lead,off", [(8, 0), (3, 0), (8, 1), (0, 3), (5, 5)])
@pytest.mark.parametrize("fmt", [None, "e4m3", "mxe5m2", "nvf4"])
def test_strides_and_alignment(fmt, lead, off):
    for dtype in ref.DTYPES:
        M, K = 5, 320
        x, res, w, h = norm_case(M, K, dtype, True, False)
        y0, h0 = mmasim.rms_norm(x.cuda(), w.cuda(), res.cuda(), fmt=fmt)
        h1 = strided(torch.zeros_like(x), lead, off)
        per_byte = 2 if fmt == "nvf4" else 1
        if fmt is None:
            out = strided(torch.zeros_like(x), lead, off)
            around = out
        else:
            n = (K + 2 * lead) // per_byte
            buf = torch.full((M * n + off,), 0xA5, dtype=torch.uint8, device="cuda")
            around = buf[off:].view(M, n)
            out = mmasim.Quantized(around[:, :K // per_byte], y0.sf.clone() if y0.sf is not None else None, y0.row_scale.clone() if y0.row_scale is not None else None)
        y1, h1b = mmasim.rms_norm(strided(x, lead, off), strided(w.view(1, -1), 0, off)[0], strided(res, lead, off), fmt=fmt, residual_out=h1, out=out)
        assert h1b is h1 and torch.equal(h1, h0)
        check_norm(y1, h1, x, res, w, h, dtype, fmt, float(np.float32(1e-6)))           # (the squares' sum has another order)
        if fmt is None:
            assert y1 is out
        else:
            assert (around[:, K // per_byte:] == 0xA5).all()
            q0, q1 = mmasim.quantize(x.cuda(), fmt), mmasim.quantize(strided(x, lead, off), fmt)
            assert all(a is b or torch.equal(a, b) for a, b in zip(q0, q1))
        dy = rows(M, K, dtype, 3)
        d1, w1 = mmasim.rms_norm_backward(strided(dy, lead, off), h1, strided(w.view(1, -1), 0, off)[0], strided(res, lead, off), dx=strided(torch.zeros_like(x), lead, off))
        check_backward(d1, w1, dy, h, w, res, dtype, float(np.float32(1e-6)))


@pytest.mark.parametrize("M,K", [(16001, 96), (9500, 128), (3001, 512), (1300, 1000), (2500, 1024), (2400, 2048), (700, 4096), (310, 14336)])
@pytest.mark.parametrize("dtype", list(ref.DTYPES))
def test_many_rows(dtype, M, K):
    """Rows of few threads with several eights each, from addresses that 16-byte accesses fit and from others; the last CTA has rows to spare."""
    x, res, w, h = norm_case(M, K, dtype, True, True)
    for fmt in ref.FORMATS:
        if K % 32 == 0 or fmt not in ("mxf4", "nvf4"):
            q = mmasim.quantize(x.cuda(), fmt)
            assert_same(q, ref.quantize(x.float().numpy(), fmt), fmt)
            assert all(a is b or torch.equal(a, b) for a, b in zip(q, mmasim.quantize(strided(x, 3, 1), fmt)))
    for fmt in [None, "e5m2", "mxe4m3"] + ["nvf4"] * (K % 32 == 0):
        y, got = mmasim.rms_norm(x.cuda(), w.cuda(), res.cuda(), fmt=fmt)
        check_norm(y, got, x, res, w, h, dtype, fmt, float(np.float32(1e-6)))
    dy = rows(M, K, dtype, 3, 0.1)
    for move in (lambda t: t.cuda(), lambda t: strided(t, 3, 1)):
        dx, dw = mmasim.rms_norm_backward(move(dy), move(h), w.cuda(), move(res))
        check_backward(dx, dw, dy, h, w, res, dtype, float(np.float32(1e-6)))


def test_rows_far_apart():
    """Offsets beyond 2^32 bytes and 2^31 elements."""
    K, ld = 64, (1 << 30) + 8
    buf = torch.zeros((2 * ld + K + 64,), dtype=torch.bfloat16, device="cuda")
    v = torch.as_strided(buf, (3, K), (ld, 1))
    x = rows(3, K, "bf16")
    v.copy_(x)
    assert_same(mmasim.quantize(v, "e4m3"), ref.quantize(x.float().numpy(), "e4m3"), "e4m3")
    y, _ = mmasim.rms_norm(v)
    want = y.clone()
    mmasim.rms_norm(v, out=v)
    assert torch.equal(v, want) and buf.count_nonzero() == want.count_nonzero()


def test_in_place():
    x, res, w, h = norm_case(6, 520, "bf16", True, False)
    y0, h0 = mmasim.rms_norm(x.cuda(), w.cuda(), res.cuda())
    xc, rc = x.cuda(), res.cuda()
    y1, h1 = mmasim.rms_norm(xc, w.cuda(), rc, residual_out=rc, out=xc)
    assert y1 is xc and h1 is rc and torch.equal(xc, y0) and torch.equal(rc, h0)
    for which in range(3):
        t = [rows(6, 520, "bf16", s).cuda() for s in (1, 2, 3)]
        want, dw = mmasim.rms_norm_backward(t[0], t[1], w.cuda(), t[2])
        dx, dw2 = mmasim.rms_norm_backward(t[0], t[1], w.cuda(), t[2], dx=t[which])
        assert dx is t[which] and torch.equal(dx, want) and torch.equal(dw, dw2)


def test_no_rows():
    x = torch.empty((0, 64), dtype=torch.bfloat16, device="cuda")
    for fmt in ref.FORMATS:
        q = mmasim.quantize(x, fmt)
        assert q.codes.shape == (0, 32 if fmt in ("mxf4", "nvf4") else 64)
    y, h = mmasim.rms_norm(x, None, x.clone(), fmt="mxe4m3")
    assert y.sf.shape == (0, 2) and h.shape == (0, 64)
    dx, dw = mmasim.rms_norm_backward(x, x, torch.ones(64, device="cuda"))
    assert dx.shape == (0, 64) and dw.dtype == torch.float32 and (dw == 0).all() and dw.shape == (64,)


def test_streams_and_graphs():
    """On a stream of the caller's, and recorded and replayed on new inputs with a second graph of the same calls in between."""
    M, K = 40, 1000
    x, res, w, _ = norm_case(M, K, "bf16", True, True)
    dy = rows(M, K, "bf16", 5)
    x, res, w, dy = (t.cuda() for t in (x, res, w, dy))
    calls = lambda x, dy, **kw: (*mmasim.rms_norm(x, w, res, fmt="e4m3", **kw), *mmasim.rms_norm_backward(dy, x, w, res, **kw), *mmasim.quantize(dy, "mxe5m2", **kw))
    flat = lambda r: [t for v in r if v is not None for t in (v if isinstance(v, tuple) else (v,)) if t is not None]
    want = flat(calls(x, dy))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = flat(calls(x, dy, stream=side))
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, got))
    graphs = []
    for _ in range(2):
        sx, sdy = torch.zeros_like(x), torch.zeros_like(dy)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            out = flat(calls(sx, sdy))
        graphs.append((graph, sx, sdy, out))
    for k in range(3):
        new = [(rows(M, K, "bf16", 20 + 2 * k + i).cuda(), rows(M, K, "bf16", 40 + 2 * k + i).cuda()) for i in range(2)]
        for (graph, sx, sdy, _), (nx, ndy) in zip(graphs, new):
            sx.copy_(nx)
            sdy.copy_(ndy)
        for graph, *_ in graphs:
            graph.replay()
        torch.cuda.synchronize()
        for (_, _, _, out), (nx, ndy) in zip(graphs, new):
            assert all(torch.equal(a, b) for a, b in zip(out, flat(calls(nx, ndy))))


def test_same_words_every_time():
    x, dy, w = rows(3000, 1111, "fp32", 1).cuda(), rows(3000, 1111, "fp32", 2).cuda(), torch.randn(1111).cuda()
    first = mmasim.rms_norm_backward(dy, x, w)
    for _ in range(5):
        again = mmasim.rms_norm_backward(dy, x, w)
        assert all(torch.equal(a, b) for a, b in zip(first, again))


def test_call_paths_agree(monkeypatch):
    """The extension module and the ctypes path in its place."""
    x, res, w, _ = norm_case(9, 96, "fp16", True, True)
    x, res, w = x.cuda(), res.cuda(), w.cuda()
    run = lambda: [*mmasim.rms_norm(x, w, res, fmt="nvf4")[0], *mmasim.rms_norm(x, w, res), *mmasim.quantize(x, "e5m2")[::2], *mmasim.rms_norm_backward(x, res, w, x)]
    fast = run()
    assert mmasim._fast is not mmasim._NoFast
    monkeypatch.setattr(mmasim, "_fast", mmasim._NoFast)
    assert all(torch.equal(a, b) for a, b in zip(fast, run()))


def test_refusals():
    x = torch.randn((4, 64), device="cuda")
    w = torch.ones(64, device="cuda")

    def refused(status, f, *a, **kw):
        with pytest.raises(mmasim.MmasimError) as e:
            f(*a, **kw)
        assert e.value.status == status, e.value

    q, n, b = mmasim.quantize, mmasim.rms_norm, mmasim.rms_norm_backward
    refused(2, q, x, "e2m1")
    refused(1, q, x.cpu(), "e4m3")
    refused(1, q, x.double(), "e4m3")
    refused(3, q, x.t(), "e4m3")
    refused(3, q, x[0], "e4m3")
    refused(3, q, x[:, :40], "nvf4")
    refused(3, q, x[:1].expand(4, 64), "e4m3")
    refused(3, q, x[:, :0], "e4m3")
    refused(3, q, torch.zeros((1, 32776), device="cuda"), "e4m3")
    refused(3, n, x, w[:60])
    refused(1, n, x, w.half())
    refused(1, n, x, w, x.half())
    refused(3, n, x, w, x[:3])
    refused(1, n, x, w, residual_out=x)
    refused(1, n, x, w, eps=-1.0)
    refused(1, n, x, w, eps=float("nan"))
    refused(2, n, x, w, fmt="e3m2")
    refused(3, n, x, w, out=torch.empty((4, 65), device="cuda"))
    buf = torch.randn((8, 64), device="cuda")
    refused(1, n, buf[:4], w, out=buf[1:5])                              # rows that others still read
    refused(1, n, x, w, buf[:4], residual_out=buf[4:], out=buf[4:])
    refused(1, n, x, buf[0], out=buf[:4])
    refused(1, q, x, "e4m3", out=mmasim.Quantized(x.view(torch.uint8)[:, :64], None, torch.empty(4, device="cuda")))
    refused(1, q, x, "e4m3", out=mmasim.Quantized(torch.empty((4, 64), dtype=torch.uint8, device="cuda"), None, None))
    refused(3, b, x, x[:3], w)
    refused(1, b, x, x.half(), w)
    refused(1, b, x[:4], buf[:4], w, dx=buf[1:5])
    wide = torch.randn((4, 128), device="cuda")                          # columns of one buffer do not meet
    y, _ = n(wide[:, :64], w, out=wide[:, 64:])
    assert torch.equal(y, n(wide[:, :64].contiguous(), w)[0])
    refused(1, n, wide[:, :64], w, out=wide[:, 60:124])
