"""Calls whose outputs would lose a gradient that autograd is asked for are refused; everything else takes parameters as they are."""
import pytest
import torch

pytestmark = pytest.mark.gpu
if torch.cuda.is_available():
    from paper_2511_10909_b200 import explore, mmasim


@pytest.fixture(params=["extension", "ctypes"])
def path(request, monkeypatch):
    mmasim.quantize(torch.zeros((1, 32), device="cuda"), "e4m3")
    if request.param == "ctypes":
        monkeypatch.setattr(mmasim, "_fast", mmasim._NoFast)


def refused(f):
    with pytest.raises(mmasim.MmasimError, match="no_grad") as e:
        f()
    assert e.value.status == 1


def test_gradients_are_not_lost_silently(path):
    x = torch.randn((4, 64), device="cuda")
    gain = torch.nn.Parameter(1 + 0.1 * torch.randn(64, device="cuda"))
    leaf = x.clone().requires_grad_()
    res = torch.randn_like(x)
    refused(lambda: mmasim.rms_norm(leaf))
    refused(lambda: mmasim.rms_norm(x, gain))
    refused(lambda: mmasim.rms_norm(x, None, leaf))
    refused(lambda: mmasim.rms_norm(x, gain.detach(), leaf, fmt="mxe4m3"))              # h is a plain output
    refused(lambda: mmasim.rms_norm(leaf, None, res, fmt="e4m3"))
    refused(lambda: mmasim.rms_norm(leaf * 2, stream=torch.cuda.current_stream()))
    w = mmasim.quantize(torch.randn((32, 64), device="cuda"), "nvf4")
    refused(lambda: mmasim.matvec4("nvf4", w.codes, w.sf, leaf, w.row_scale))
    refused(lambda: mmasim.matvec4("nvf4", w.codes, w.sf, x, w.row_scale.clone().requires_grad_()))
    with torch.no_grad():
        y, h = mmasim.rms_norm(leaf, gain, res)
        z = mmasim.matvec4("nvf4", w.codes, w.sf, leaf, w.row_scale)
    want, want_h = mmasim.rms_norm(x, gain.detach(), res)
    assert torch.equal(y, want) and torch.equal(h, want_h) and not y.requires_grad
    assert torch.equal(z, mmasim.matvec4("nvf4", w.codes, w.sf, x, w.row_scale))


def test_codes_and_gradients_take_parameters(path):
    x = torch.randn((4, 64), device="cuda")
    gain, leaf = torch.nn.Parameter(torch.ones(64, device="cuda")), x.clone().requires_grad_()
    same = lambda a, b: all(s is t or torch.equal(s, t) for s, t in zip(a, b))
    for fmt in mmasim.QUANTIZED_FORMATS:
        assert same(mmasim.quantize(leaf, fmt), mmasim.quantize(x, fmt))
        assert same(mmasim.rms_norm(leaf, gain, fmt=fmt)[0], mmasim.rms_norm(x, gain.detach(), fmt=fmt)[0])
        assert same(mmasim.rms_norm(x, gain, x, fmt=fmt)[0], mmasim.rms_norm(x, gain.detach(), x, fmt=fmt)[0])
    assert same(mmasim.rms_norm_backward(x, leaf, gain), mmasim.rms_norm_backward(x, x, gain.detach()))


def test_a_layer_of_parameters():
    g = torch.Generator().manual_seed(1)
    x, W = (torch.randn(s, generator=g).cuda().requires_grad_() for s in ((8, 64), (32, 64)))
    gain = torch.nn.Parameter(torch.ones(64, device="cuda"))
    rows = (("blackwell", "nvf4"),)
    assert explore.quantised_layer(x, gain, W, rows, residual=x) == explore.quantised_layer(x.detach(), gain.detach(), W.detach(), rows, residual=x.detach())
