"""Every kernel that the operators on rows and the 4-bit products are compiled into is one that some call launches: calls over sizes, types and
alignments on the host, the runtime's launch a stand-in that notes the kernel, against the kernels in the library."""
import re
import subprocess

from helpers import host_program

PROGRAM = r"""
#include <cstdio>
#include <cstring>
#include <set>
#include <cuda.h>
#include <cuda_runtime.h>
#include <dlfcn.h>
#include "mmasim_internal.h"
#define SHOWN extern "C" __attribute__((visibility("default")))
static std::set<const void*> seen;
SHOWN cudaError_t cudaLaunchKernelExC(const cudaLaunchConfig_t*, const void* f, void**) { seen.insert(f); return cudaSuccess; }
SHOWN cudaError_t cudaGetLastError() { return cudaSuccess; }
SHOWN cudaError_t cudaFuncSetAttribute(const void*, cudaFuncAttribute, int) { return cudaSuccess; }
SHOWN cudaError_t cudaGetDevice(int* d) { *d = 0; return cudaSuccess; }
SHOWN cudaError_t cudaPointerGetAttributes(cudaPointerAttributes* a, const void*) {
    std::memset(a, 0, sizeof(*a));
    a->type = cudaMemoryTypeDevice;
    return cudaSuccess;
}
static char* at(long long x) { return reinterpret_cast<char*>(x << 44); }
int main() {
    const int types[] = {MMASIM_F32, MMASIM_BF16, MMASIM_F16};
    const int outs[] = {MMASIM_E4M3, MMASIM_E5M2, MMASIM_MXE4M3, MMASIM_MXE5M2, MMASIM_MXF4_GST, MMASIM_NVF4_GST};
    const int lengths[] = {1, 8, 32, 33, 64, 96, 128, 256, 512, 1000, 1024, 1111, 1536, 2048, 2080, 4096, 4128, 6144, 8192, 9600, 12288, 16384, 16416, 20480, 20500, 28672, 32736, 32768};
    const long long rows[] = {1, 200, 300, 2000, 20000, 300000};
    char *X = at(1), *R = at(2), *H = at(3), *O = at(4), *W = at(5), *S = at(6), *D = at(7);
    float* RS = reinterpret_cast<float*>(at(8));
    bool ok = true;
    for (int type : types)
        for (int K : lengths)
            for (int off = 0; off < 8; off += 4) {              // bytes behind a multiple of 16
                for (long long M : rows) {
                    for (int out : outs) {
                        const bool four = out == MMASIM_MXF4_GST || out == MMASIM_NVF4_GST;
                        if (four && K % 32) continue;
                        void* sf = out == MMASIM_E4M3 || out == MMASIM_E5M2 ? nullptr : S;
                        float* rs = out == MMASIM_E4M3 || out == MMASIM_E5M2 || out == MMASIM_NVF4_GST ? RS : nullptr;
                        ok &= mmasim_quantize(type, out, M, K, X + off, 0, O, 0, sf, rs, nullptr) == MMASIM_OK;
                        mmasim_rms_norm_args n = {};
                        n.x = X + off; n.weight = W; n.weight_fmt = MMASIM_F32; n.out = O; n.out_fmt = out; n.sf = sf; n.row_scale = rs;
                        ok &= mmasim_rms_norm(type, M, K, &n, nullptr) == MMASIM_OK;
                    }
                    mmasim_rms_norm_args n = {};
                    n.x = X + off; n.residual = R; n.residual_out = H; n.weight = W; n.weight_fmt = MMASIM_F32; n.out = O; n.out_fmt = type;
                    ok &= mmasim_rms_norm(type, M, K, &n, nullptr) == MMASIM_OK;
                    mmasim_rms_norm_backward_args b = {};
                    b.dy = X + off; b.h = H; b.weight = W; b.weight_fmt = MMASIM_F32; b.dx = O; b.dweight = D; b.workspace = S;
                    b.workspace_bytes = mmasim_rms_norm_backward_workspace(M, K);
                    ok &= mmasim_rms_norm_backward(type, M, K, &b, nullptr) == MMASIM_OK;
                }
                if (K % 32 || (type == MMASIM_F32 && K > 20480)) continue;
                for (int T = 1; T <= 17; ++T)
                    for (int w : {MMASIM_MXF4_GST, MMASIM_NVF4_GST})
                        ok &= mmasim_matvec4(w, type, T, 100, K, W, 0, S, RS, X + off, 0, O, 0, nullptr) == MMASIM_OK;
            }
    std::printf("%d\n", int(ok));
    for (const void* f : seen) {
        Dl_info info;
        dladdr(f, &info);
        std::printf("%llx\n", (unsigned long long)(static_cast<const char*>(f) - static_cast<const char*>(info.dli_fbase)));
    }
}
"""


def test_every_kernel_is_launched_by_some_call(tmp_path):
    from paper_2511_10909_b200.build import build
    ok, *launched = host_program(tmp_path, PROGRAM)()
    assert ok == "1"
    launched = {int(x, 16) for x in launched}
    names = {}
    for line in subprocess.run(["nm", "-C", build()], check=True, capture_output=True, text=True).stdout.splitlines():
        found = re.match(r"([0-9a-f]+) [tTwW] .*\b((?:rows|backward|backward_ring|dweight|matvec4)_kernel<.*>)\(", line)
        if found and "__device_stub__" not in line:
            names[int(found.group(1), 16)] = found.group(2)
    assert len(names) > 200 and launched <= set(names)
    assert not {n for a, n in names.items() if a not in launched}
