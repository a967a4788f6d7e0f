"""Arguments that mmasim_quantize, mmasim_rms_norm, mmasim_rms_norm_backward and mmasim_matvec4 refuse or take, on the host: the runtime's
answers about pointers and its launch are stand-ins of the program, nothing reaches a GPU.  And the formulas that the GPU tests hold the
kernels to, against automatic differentiation in 64 bits."""
import numpy as np
import pytest
import torch

import rows_ref as ref
from helpers import host_program

PROGRAM = r"""
#include <cstdio>
#include <cstring>
#include <cuda.h>
#include <cuda_runtime.h>
#include "mmasim_internal.h"
#define SHOWN extern "C" __attribute__((visibility("default")))
static int launches = 0, device = 0, host_from = 0;
SHOWN cudaError_t cudaLaunchKernelExC(const cudaLaunchConfig_t*, const void*, void**) { ++launches; return cudaSuccess; }
SHOWN cudaError_t cudaGetLastError() { return cudaSuccess; }
SHOWN cudaError_t cudaFuncSetAttribute(const void*, cudaFuncAttribute, int) { return cudaSuccess; }
SHOWN cudaError_t cudaGetDevice(int* d) { *d = 0; return cudaSuccess; }
SHOWN cudaError_t cudaPointerGetAttributes(cudaPointerAttributes* a, const void* p) {
    std::memset(a, 0, sizeof(*a));
    a->type = reinterpret_cast<uintptr_t>(p) < 0x10000 ? cudaMemoryTypeUnregistered : cudaMemoryTypeDevice;
    a->device = reinterpret_cast<uintptr_t>(p) >= 0x7000000000 ? 1 : 0;
    return cudaSuccess;
}
static CUresult encode(CUtensorMap*, ...) { return CUDA_SUCCESS; }
SHOWN cudaError_t cudaGetDriverEntryPoint(const char*, void** f, unsigned long long, cudaDriverEntryPointQueryResult* found) {
    *f = reinterpret_cast<void*>(encode);
    *found = cudaDriverEntryPointSuccess;
    return cudaSuccess;
}
static char* at(long long x) { return reinterpret_cast<char*>(x); }
static void show(const char* what, int st) { std::printf("%s %d %d\n", what, st, launches); launches = 0; }
int main() {
    char *X = at(0x100000), *R = at(0x200000), *H = at(0x300000), *O = at(0x400000), *W = at(0x500000), *S = at(0x600000);
    float* RS = reinterpret_cast<float*>(at(0x700000));
    auto quant = [&](const char* n, int in, int out, long long M, long long K, void* x, long long ldx, void* c, long long ldc, void* sf, float* rs) {
        show(n, mmasim_quantize(in, out, M, K, x, ldx, c, ldc, sf, rs, nullptr));
    };
    quant("row", MMASIM_BF16, MMASIM_E4M3, 4, 100, X, 0, O, 0, nullptr, RS);
    quant("mx", MMASIM_F32, MMASIM_MXE5M2, 4, 33, X, 40, O, 64, S, nullptr);
    quant("nv", MMASIM_F16, MMASIM_NVF4_GST, 4, 64, X, 0, O, 0, S, RS);
    quant("no_rows", MMASIM_F16, MMASIM_NVF4_GST, 0, 64, nullptr, 0, nullptr, 0, nullptr, nullptr);
    quant("in_fmt", MMASIM_F64, MMASIM_E4M3, 4, 64, X, 0, O, 0, nullptr, RS);
    quant("out_fmt", MMASIM_F32, MMASIM_E2M1, 4, 64, X, 0, O, 0, nullptr, RS);
    quant("plain", MMASIM_F32, MMASIM_F32, 4, 64, X, 0, O, 0, nullptr, nullptr);
    quant("fp4_k", MMASIM_F32, MMASIM_MXF4_GST, 4, 48, X, 0, O, 0, S, nullptr);
    quant("fp4_odd_ld", MMASIM_F32, MMASIM_MXF4_GST, 4, 64, X, 0, O, 65, S, nullptr);
    quant("negative", MMASIM_F32, MMASIM_E4M3, -1, 64, X, 0, O, 0, nullptr, RS);
    quant("k0", MMASIM_F32, MMASIM_E4M3, 4, 0, X, 0, O, 0, nullptr, RS);
    quant("k_most", MMASIM_F32, MMASIM_E4M3, 4, 32768, X, 0, O, 0, nullptr, RS);
    quant("k_more", MMASIM_F32, MMASIM_E4M3, 4, 32769, X, 0, O, 0, nullptr, RS);
    quant("ld", MMASIM_F32, MMASIM_E4M3, 4, 64, X, 63, O, 0, nullptr, RS);
    quant("no_scale", MMASIM_F32, MMASIM_E4M3, 4, 64, X, 0, O, 0, nullptr, nullptr);
    quant("sf_for_row", MMASIM_F32, MMASIM_E4M3, 4, 64, X, 0, O, 0, S, RS);
    quant("odd_address", MMASIM_BF16, MMASIM_E4M3, 4, 64, X + 1, 0, O, 0, nullptr, RS);
    quant("host", MMASIM_BF16, MMASIM_E4M3, 4, 64, at(0x1000), 0, O, 0, nullptr, RS);
    quant("other_device", MMASIM_BF16, MMASIM_E4M3, 4, 64, at(0x7000000000), 0, O, 0, nullptr, RS);
    quant("over", MMASIM_BF16, MMASIM_E4M3, 4, 64, X, 0, X + 511, 0, nullptr, RS);
    quant("behind", MMASIM_BF16, MMASIM_E4M3, 4, 64, X, 0, X + 512, 0, nullptr, RS);
    quant("same", MMASIM_BF16, MMASIM_E4M3, 4, 64, X, 0, X, 0, nullptr, RS);
    quant("columns", MMASIM_BF16, MMASIM_E4M3, 4, 64, X, 128, X + 128, 256, nullptr, RS);          // codes in the gaps of x
    quant("columns_meet", MMASIM_BF16, MMASIM_E4M3, 4, 64, X, 128, X + 127, 256, nullptr, RS);
    quant("columns_wrap", MMASIM_BF16, MMASIM_E4M3, 4, 64, X, 128, X - 64, 256, nullptr, RS);      // the gap in front of x
    quant("columns_wrap_meet", MMASIM_BF16, MMASIM_E4M3, 4, 64, X, 128, X - 63, 256, nullptr, RS);

    mmasim_rms_norm_args n;
    auto fresh = [&] {
        std::memset(&n, 0, sizeof(n));
        n.x = X; n.residual = R; n.residual_out = H; n.weight = W; n.weight_fmt = MMASIM_BF16; n.out = O; n.out_fmt = MMASIM_BF16; n.eps = 1e-6f;
    };
    auto norm = [&](const char* name) { show(name, mmasim_rms_norm(MMASIM_BF16, 4, 64, &n, nullptr)); fresh(); };
    fresh(); norm("norm");
    n.residual_out = R; n.out = X; norm("norm_in_place");
    n.residual_out = X; n.out = R; norm("norm_crossed");
    n.out = H; norm("norm_out_over_residual_out");
    n.residual_out = nullptr; norm("norm_half_residual");
    n.weight_fmt = MMASIM_F16; norm("norm_weight_type");
    n.weight_fmt = MMASIM_F32; norm("norm_weight_f32");
    n.weight = nullptr; n.residual = nullptr; n.residual_out = nullptr; norm("norm_bare");
    n.out = W; norm("norm_over_weight");
    n.out_fmt = MMASIM_E4M3; n.row_scale = RS; norm("norm_e4m3");
    n.out_fmt = MMASIM_E4M3; n.row_scale = RS; n.out = X; norm("norm_e4m3_over_x");
    n.out_fmt = MMASIM_F32; norm("norm_f32_out");
    n.row_scale = RS; norm("norm_plain_scale");
    n.eps = -1.0f; norm("norm_eps");
    n.out = X + 128; norm("norm_shifted_rows");
    show("norm_null", mmasim_rms_norm(MMASIM_BF16, 4, 64, nullptr, nullptr));

    mmasim_rms_norm_backward_args b;
    auto freshb = [&] {
        std::memset(&b, 0, sizeof(b));
        b.dy = X; b.h = H; b.weight = W; b.dresidual = R; b.dx = O; b.dweight = S; b.workspace = RS; b.weight_fmt = MMASIM_BF16; b.eps = 1e-6f;
        b.workspace_bytes = mmasim_rms_norm_backward_workspace(4, 64);
    };
    auto back = [&](const char* name) { show(name, mmasim_rms_norm_backward(MMASIM_BF16, 4, 64, &b, nullptr)); freshb(); };
    freshb(); back("back");
    b.dx = X; back("back_dx_is_dy");
    b.dx = H; back("back_dx_is_h");
    b.dx = X + 2; back("back_dx_shifted");
    b.workspace_bytes -= 1; back("back_small_workspace");
    b.workspace = nullptr; back("back_no_workspace");
    b.dweight = nullptr; b.workspace = nullptr; back("back_no_dweight");
    b.dweight = W; back("back_dweight_over_weight");
    b.workspace = O; back("back_workspace_over_dx");
    b.weight_fmt = MMASIM_F16; back("back_weight_type");
    b.h = nullptr; back("back_no_h");
    show("back_no_rows", mmasim_rms_norm_backward(MMASIM_BF16, 0, 64, &b, nullptr));
    std::printf("workspace %d %d %d\n", int(mmasim_rms_norm_backward_workspace(-1, 64)), int(mmasim_rms_norm_backward_workspace(4, 32769)), int(mmasim_rms_norm_backward_workspace(0, 64)));

    auto mat = [&](const char* name, int wf, int f, long long T, long long N, long long K, void* w, long long ldw, void* sf, float* rs, void* x, void* y) {
        show(name, mmasim_matvec4(wf, f, T, N, K, w, ldw, sf, rs, x, 0, y, 0, nullptr));
    };
    mat("mat", MMASIM_NVF4_GST, MMASIM_BF16, 1, 16, 64, W, 0, S, RS, X, O);
    mat("mat_no_scale", MMASIM_MXF4_GST, MMASIM_F32, 1, 16, 64, W, 96, S, nullptr, X, O);
    mat("mat_no_tokens", MMASIM_MXF4_GST, MMASIM_F32, 0, 16, 64, nullptr, 0, nullptr, nullptr, nullptr, nullptr);
    mat("mat_fmt", MMASIM_E4M3, MMASIM_BF16, 1, 16, 64, W, 0, S, RS, X, O);
    mat("mat_type", MMASIM_NVF4_GST, MMASIM_F64, 1, 16, 64, W, 0, S, RS, X, O);
    mat("mat_k", MMASIM_NVF4_GST, MMASIM_BF16, 1, 16, 48, W, 0, S, RS, X, O);
    mat("mat_k_f32", MMASIM_NVF4_GST, MMASIM_F32, 2, 16, 20480, W, 0, S, RS, X, O);
    mat("mat_k_f32_more", MMASIM_NVF4_GST, MMASIM_F32, 1, 16, 20512, W, 0, S, RS, X, O);
    mat("mat_k_most", MMASIM_NVF4_GST, MMASIM_BF16, 3, 16, 32768, W, 0, S, RS, X, O);
    mat("mat_k_more", MMASIM_NVF4_GST, MMASIM_BF16, 1, 16, 32800, W, 0, S, RS, X, O);
    mat("mat_n", MMASIM_NVF4_GST, MMASIM_BF16, 1, 0, 64, W, 0, S, RS, X, O);
    mat("mat_ld", MMASIM_NVF4_GST, MMASIM_BF16, 1, 16, 64, W, 72, S, RS, X, O);
    mat("mat_align", MMASIM_NVF4_GST, MMASIM_BF16, 1, 16, 64, W + 8, 0, S, RS, X, O);
    mat("mat_sf_align", MMASIM_NVF4_GST, MMASIM_BF16, 1, 16, 64, W, 0, S + 1, RS, X, O);
    mat("mat_sf_bytes", MMASIM_MXF4_GST, MMASIM_BF16, 1, 16, 64, W, 0, S + 1, nullptr, X, O);
    mat("mat_over", MMASIM_NVF4_GST, MMASIM_BF16, 1, 64, 64, W, 0, S, RS, X, X);
    mat("mat_null", MMASIM_NVF4_GST, MMASIM_BF16, 1, 16, 64, W, 0, nullptr, RS, X, O);
}
"""

OK, ARG, UNSUPPORTED, SHAPE, ALIGN = 0, 1, 2, 3, 4
WANT = dict(row=OK, mx=OK, nv=OK, no_rows=OK, in_fmt=ARG, out_fmt=UNSUPPORTED, plain=UNSUPPORTED, fp4_k=SHAPE, fp4_odd_ld=SHAPE, negative=SHAPE, k0=SHAPE, k_most=OK,
            k_more=SHAPE, ld=SHAPE, no_scale=ARG, sf_for_row=ARG, odd_address=ALIGN, host=ARG, other_device=ARG, over=ARG, behind=OK, same=ARG, columns=OK,
            columns_meet=ARG, columns_wrap=OK, columns_wrap_meet=ARG, norm=OK, norm_in_place=OK, norm_crossed=OK, norm_out_over_residual_out=ARG, norm_half_residual=ARG,
            norm_weight_type=ARG, norm_weight_f32=OK, norm_bare=OK, norm_over_weight=ARG, norm_e4m3=OK, norm_e4m3_over_x=ARG, norm_f32_out=UNSUPPORTED,
            norm_plain_scale=ARG, norm_eps=ARG, norm_shifted_rows=ARG, norm_null=ARG, back=OK, back_dx_is_dy=OK, back_dx_is_h=OK, back_dx_shifted=ARG,
            back_small_workspace=ARG, back_no_workspace=ARG, back_no_dweight=OK, back_dweight_over_weight=ARG, back_workspace_over_dx=ARG, back_weight_type=ARG,
            back_no_h=ARG, back_no_rows=OK, mat=OK, mat_no_scale=OK, mat_no_tokens=OK, mat_fmt=UNSUPPORTED, mat_type=ARG, mat_k=SHAPE, mat_k_f32=OK, mat_k_f32_more=SHAPE, mat_k_most=OK, mat_k_more=SHAPE, mat_n=SHAPE, mat_ld=ALIGN,
            mat_align=ALIGN, mat_sf_align=ALIGN, mat_sf_bytes=OK, mat_over=ARG, mat_null=ARG)


def test_what_the_calls_refuse(tmp_path):
    lines = host_program(tmp_path, PROGRAM)()
    got = {line.split()[0]: tuple(map(int, line.split()[1:])) for line in lines}
    assert got.pop("workspace") == (0, 0, 0)
    assert {k: v[0] for k, v in got.items()} == WANT
    for name, (status, launched) in got.items():
        none = status or name in ("no_rows", "mat_no_tokens")
        assert (launched == 0) == bool(none), name
    assert got["back"][1] == 2 and got["back_no_dweight"][1] == 1 and got["back_no_rows"][1] == 1


def test_cpu_tensors_are_refused():
    from paper_2511_10909_b200 import mmasim
    x = torch.zeros((2, 32))
    for call in (lambda: mmasim.quantize(x, "e4m3"), lambda: mmasim.rms_norm(x), lambda: mmasim.rms_norm_backward(x, x),
                 lambda: mmasim.matvec4("mxf4", x.to(torch.uint8), x.to(torch.uint8), x)):
        with pytest.raises(mmasim.MmasimError) as e:
            call()
        assert e.value.status == 1


@pytest.mark.parametrize("weighted", [False, True])
def test_gradient_formula(weighted):
    """rows_ref's gradients against automatic differentiation and against differences, in 64 bits."""
    g = torch.Generator().manual_seed(1)
    x, dy, dh = (torch.randn((3, 20), generator=g, dtype=torch.float64) for _ in range(3))
    w = torch.randn(20, generator=g, dtype=torch.float64) if weighted else torch.ones(20, dtype=torch.float64)
    x.requires_grad_()
    w.requires_grad_()
    loss = lambda x, w: ((x / torch.sqrt((x * x).mean(1, keepdim=True) + 1e-3) * w) * dy + x * dh).sum()
    loss(x, w).backward()
    dx, dw, _, _ = ref.rms_norm_backward(dy.numpy(), x.detach().numpy(), w.detach().numpy() if weighted else None, dh.numpy(), 1e-3)
    assert np.allclose(dx, x.grad.numpy(), rtol=1e-12, atol=1e-13) and np.allclose(dw, w.grad.numpy(), rtol=1e-12, atol=1e-13)
    d, step = torch.randn((3, 20), generator=g, dtype=torch.float64), 1e-5
    num = (loss(x.detach() + step * d, w.detach()) - loss(x.detach() - step * d, w.detach())) / (2 * step)
    assert abs(num.item() - (dx * d.numpy()).sum()) < 1e-7


def test_reference_casts():
    """rows_ref.quantize's codes stand for the nearest values (torch's casts as the witness)."""
    x = torch.randn((8, 96), generator=torch.Generator().manual_seed(2)) * 3
    for fmt, kind in (("e4m3", torch.float8_e4m3fn), ("e5m2", torch.float8_e5m2)):
        codes, _, s = ref.quantize(x.numpy(), fmt)
        assert np.array_equal(codes, (x / torch.from_numpy(s)[:, None]).to(kind).view(torch.uint8).numpy())
    for fmt in ref.FORMATS:
        q = ref.quantize(x.numpy(), fmt)
        ref.assert_quantised(q, x.double().numpy(), fmt, 0.0)
        assert np.array_equal(ref.unpack(ref.pack(q[0], fmt), fmt), q[0])
