// C ABI of the operators around products of scaled operands: argument checks, then the kernels' launchers.
#include <cstring>
#include "mmasim_rows.cuh"

namespace mmasim {
namespace {

int element_fmt(int fmt) { return fmt == MMASIM_F32 ? EF_F32 : fmt == MMASIM_BF16 ? EF_BF16 : fmt == MMASIM_F16 ? EF_F16 : -1; }
int element_bytes(int fmt) { return fmt == MMASIM_F32 ? 4 : 2; }
bool quantised(int fmt) {
    return fmt == MMASIM_E4M3 || fmt == MMASIM_E5M2 || fmt == MMASIM_MXE4M3 || fmt == MMASIM_MXE5M2 || fmt == MMASIM_MXF4_GST || fmt == MMASIM_NVF4_GST;
}
bool packed4(int fmt) { return fmt == MMASIM_MXF4_GST || fmt == MMASIM_NVF4_GST; }
bool has_row_scale(int fmt) { return fmt == MMASIM_E4M3 || fmt == MMASIM_E5M2 || fmt == MMASIM_NVF4_GST; }
int block_of(int fmt) { return fmt == MMASIM_NVF4_GST ? 16 : (fmt == MMASIM_E4M3 || fmt == MMASIM_E5M2 ? 0 : 32); }

// One argument: `rows` rows of `len` bytes, `pitch` bytes apart.
struct Span {
    const char* name;
    const void* p;
    int64_t rows, len, pitch;
};
bool same_rows(const Span& a, const Span& b) { return a.p == b.p && a.pitch == b.pitch; }
bool meet(const Span& a, const Span& b) {
    if (!a.p || !b.p || a.rows < 1 || b.rows < 1) return false;
    const uintptr_t p = reinterpret_cast<uintptr_t>(a.p), q = reinterpret_cast<uintptr_t>(b.p);
    const uintptr_t p_end = p + uintptr_t((a.rows - 1) * a.pitch + a.len), q_end = q + uintptr_t((b.rows - 1) * b.pitch + b.len);
    if (p >= q_end || q >= p_end) return false;
    if (a.pitch != b.pitch || a.rows == 1 || b.rows == 1) return true;
    // columns of one buffer lie between each other's rows
    const uintptr_t pitch = uintptr_t(a.pitch), off = p < q ? (q - p) % pitch : (pitch - (p - q) % pitch) % pitch;      // b's rows behind a's
    return !(off >= uintptr_t(a.len) && pitch - off >= uintptr_t(b.len));
}
// MMASIM_OK if p is memory of the current device, aligned to `align` bytes.
int check_span(const char* call, const Span& s, int align, int device) {
    if (!s.p) return MMASIM_OK;
    if (reinterpret_cast<uintptr_t>(s.p) % uintptr_t(align)) { set_error("%s: %s must be aligned to %d bytes", call, s.name, align); return MMASIM_ERR_ALIGN; }
    cudaPointerAttributes attr;
    const cudaError_t err = cudaPointerGetAttributes(&attr, s.p);
    if (err != cudaSuccess) {
        cudaGetLastError();
        set_error("%s: cudaPointerGetAttributes(%s) failed: %s", call, s.name, cudaGetErrorString(err));
        return MMASIM_ERR_CUDA;
    }
    if (attr.type == cudaMemoryTypeManaged) return MMASIM_OK;
    if (attr.type != cudaMemoryTypeDevice) { set_error("%s: %s is not a device pointer", call, s.name); return MMASIM_ERR_INVALID_ARG; }
    if (attr.device != device) { set_error("%s: %s is on device %d, the current one is %d", call, s.name, attr.device, device); return MMASIM_ERR_INVALID_ARG; }
    return MMASIM_OK;
}
int current_device(const char* call, int* device) {
    const cudaError_t err = cudaGetDevice(device);
    if (err == cudaSuccess) return MMASIM_OK;
    cudaGetLastError();
    set_error("%s: %s", call, cudaGetErrorString(err));
    return MMASIM_ERR_CUDA;
}
// Leading dimensions: 0 = packed, else at least K and a row's length in bytes that fits.
int check_ld(const char* call, const char* name, int64_t* ld, int64_t K) {
    if (!*ld) *ld = K;
    if (*ld < K || *ld > (int64_t(1) << 40)) { set_error("%s: leading dimension of %s is %lld, a row has %lld elements", call, name, (long long)*ld, (long long)K); return MMASIM_ERR_SHAPE; }
    return MMASIM_OK;
}
int check_shape(const char* call, int64_t M, int64_t K, int64_t most_k) {
    if (M < 0 || M > 0x7FFFFFFF) { set_error("%s: %lld rows, from 0 to 2^31 - 1 are taken", call, (long long)M); return MMASIM_ERR_SHAPE; }
    if (K < 1 || K > most_k) { set_error("%s: rows of %lld elements, from 1 to %lld are taken", call, (long long)K, (long long)most_k); return MMASIM_ERR_SHAPE; }
    return MMASIM_OK;
}
// Rules on a quantised output that mmasim_quantize and mmasim_rms_norm share.
int check_output(const char* call, int out_fmt, int64_t K, int64_t ld_out, const void* sf, const void* row_scale) {
    if (packed4(out_fmt) && (K % 32 || ld_out % 2)) { set_error("%s: 4-bit codes need K a multiple of 32 and an even leading dimension", call); return MMASIM_ERR_SHAPE; }
    if ((sf != nullptr) != (block_of(out_fmt) != 0)) { set_error("%s: the format %s sf", call, block_of(out_fmt) ? "needs" : "has no"); return MMASIM_ERR_INVALID_ARG; }
    if ((row_scale != nullptr) != has_row_scale(out_fmt)) { set_error("%s: the format %s row_scale", call, has_row_scale(out_fmt) ? "needs" : "has no"); return MMASIM_ERR_INVALID_ARG; }
    return MMASIM_OK;
}
// Rows in, rows or codes out: mmasim_rms_norm, and mmasim_quantize as one without the norm.
int run_rows(const char* call, int fmt, int64_t M, int64_t K, mmasim_rms_norm_args p, bool norm, void* stream) {
    if (element_fmt(fmt) < 0) { set_error("%s: rows are FP32, BF16 or FP16", call); return MMASIM_ERR_INVALID_ARG; }
    if (!quantised(p.out_fmt) && !(norm && p.out_fmt == fmt)) {
        set_error("%s: the output format is %sE4M3, E5M2, MXE4M3, MXE5M2, MXF4_GST or NVF4_GST", call, norm ? "the rows' own, or " : "");
        return MMASIM_ERR_UNSUPPORTED;
    }
    if (p.weight && p.weight_fmt != fmt && p.weight_fmt != MMASIM_F32) { set_error("%s: the weight is of the rows' type or FP32", call); return MMASIM_ERR_INVALID_ARG; }
    if (!(p.eps >= 0.0f)) { set_error("%s: eps must be >= 0", call); return MMASIM_ERR_INVALID_ARG; }
    int st = check_shape(call, M, K, ROWS_MAX_K);
    if (st == MMASIM_OK) st = check_ld(call, "x", &p.ldx, K);
    if (st == MMASIM_OK) st = check_ld(call, "residual", &p.ld_residual, K);
    if (st == MMASIM_OK) st = check_ld(call, "residual_out", &p.ld_residual_out, K);
    if (st == MMASIM_OK) st = check_ld(call, "out", &p.ld_out, K);
    if (st != MMASIM_OK) return st;
    if (M == 0) return MMASIM_OK;
    if (!p.x || !p.out) { set_error("%s: x and the output must not be NULL", call); return MMASIM_ERR_INVALID_ARG; }
    if ((p.residual != nullptr) != (p.residual_out != nullptr)) { set_error("%s: residual and residual_out must be given together", call); return MMASIM_ERR_INVALID_ARG; }
    const bool plain = !quantised(p.out_fmt);
    if (plain && (p.sf || p.row_scale)) { set_error("%s: a plain output has no scales", call); return MMASIM_ERR_INVALID_ARG; }
    if (!plain && (st = check_output(call, p.out_fmt, K, p.ld_out, p.sf, p.row_scale)) != MMASIM_OK) return st;
    const int b = element_bytes(fmt), kb = block_of(p.out_fmt);
    const int64_t out_len = plain ? K * b : (packed4(p.out_fmt) ? K / 2 : K), out_pitch = plain ? p.ld_out * b : (packed4(p.out_fmt) ? p.ld_out / 2 : p.ld_out);
    const Span x = {"x", p.x, M, K * b, p.ldx * b}, r = {"residual", p.residual, M, K * b, p.ld_residual * b},
               w = {"weight", p.weight, 1, K * (p.weight_fmt == MMASIM_F32 ? 4 : 2), 0}, h = {"residual_out", p.residual_out, M, K * b, p.ld_residual_out * b},
               o = {plain ? "out" : "codes", p.out, M, out_len, out_pitch}, sf = {"sf", p.sf, 1, kb ? M * ((K + kb - 1) / kb) : 0, 0},
               rs = {"row_scale", p.row_scale, 1, M * 4, 0};
    int device = 0;
    if ((st = current_device(call, &device)) != MMASIM_OK) return st;
    const Span* all[] = {&x, &r, &w, &h, &o, &sf, &rs};
    const int align[] = {b, b, p.weight_fmt == MMASIM_F32 ? 4 : 2, b, plain ? b : 1, 1, 4};
    for (int i = 0; i < 7; ++i)
        if ((st = check_span(call, *all[i], align[i], device)) != MMASIM_OK) return st;
    for (int i = 3; i < 7; ++i)             // every output against everything in front of it
        for (int j = 0; j < i; ++j) {
            const bool in_place = (i == 3 || (i == 4 && plain)) && j < 2 && same_rows(*all[i], *all[j]);
            if (!in_place && meet(*all[i], *all[j])) { set_error("%s: %s lies over %s", call, all[i]->name, all[j]->name); return MMASIM_ERR_INVALID_ARG; }
        }
    return launch_rows(element_fmt(fmt), M, K, p, norm, static_cast<cudaStream_t>(stream));
}

}  // namespace

int launch_rows(int fmt, int64_t M, int64_t K, const mmasim_rms_norm_args& p, bool norm, cudaStream_t stream) {
    const int bytes = fmt == EF_F32 ? 4 : 2;
    auto vec = [](const void* q, int64_t pitch, int to) { return int((reinterpret_cast<uintptr_t>(q) | uintptr_t(pitch)) % to == 0); };
    rows::Args a;
    std::memset(&a, 0, sizeof(a));
    a.M = M; a.K = int(K);
    a.x = p.x; a.residual = p.residual; a.w = p.weight; a.h_out = p.residual_out; a.out = p.out;
    a.sf = static_cast<uint8_t*>(p.sf);
    a.row_scale = p.row_scale;
    a.ldx = p.ldx; a.ldr = p.ld_residual; a.ldh = p.ld_residual_out; a.ldo = p.ld_out;
    a.eps = p.eps;
    a.e5m2 = p.out_fmt == MMASIM_E5M2 || p.out_fmt == MMASIM_MXE5M2;
    a.w_f32 = p.weight_fmt == MMASIM_F32;
    a.vec_x = vec(p.x, a.ldx * bytes, 16); a.vec_r = vec(p.residual, a.ldr * bytes, 16); a.vec_h = vec(p.residual_out, a.ldh * bytes, 16);
    a.vec_w = vec(p.weight, 0, 16);
    int out = rows::OUT_PLAIN;
    if (p.out_fmt == MMASIM_E4M3 || p.out_fmt == MMASIM_E5M2) out = rows::OUT_FP8;
    else if (p.out_fmt == MMASIM_MXE4M3 || p.out_fmt == MMASIM_MXE5M2) out = rows::OUT_MX8;
    else if (p.out_fmt == MMASIM_MXF4_GST) out = rows::OUT_MXF4;
    else if (p.out_fmt == MMASIM_NVF4_GST) out = rows::OUT_NVF4;
    a.vec_o = out == rows::OUT_PLAIN ? vec(p.out, a.ldo * bytes, 16) : packed4(p.out_fmt) ? vec(p.out, a.ldo / 2, 4) : vec(p.out, a.ldo, 8);
    if (const int kb = block_of(p.out_fmt)) a.ld_sf = (K + kb - 1) / kb;
    const cudaError_t err = fmt == EF_F32 ? rows::launch_f32(a, out, norm, stream) : fmt == EF_BF16 ? rows::launch_bf16(a, out, norm, stream) : rows::launch_f16(a, out, norm, stream);
    if (err != cudaSuccess) { set_error("%s: %s", norm ? "mmasim_rms_norm" : "mmasim_quantize", cudaGetErrorString(err)); return MMASIM_ERR_CUDA; }
    return MMASIM_OK;
}

}  // namespace mmasim

using namespace mmasim;

extern "C" {

int mmasim_quantize(int in_fmt, int out_fmt, int64_t M, int64_t K, const void* x, int64_t ldx, void* codes, int64_t ld_codes, void* sf,
                    float* row_scale, void* stream) {
    mmasim_rms_norm_args p;
    std::memset(&p, 0, sizeof(p));
    p.x = x; p.ldx = ldx;
    p.out = codes; p.ld_out = ld_codes;
    p.sf = sf; p.row_scale = row_scale;
    p.out_fmt = out_fmt;
    return run_rows("mmasim_quantize", in_fmt, M, K, p, false, stream);
}

int mmasim_rms_norm(int fmt, int64_t M, int64_t K, const mmasim_rms_norm_args* args, void* stream) {
    if (!args) { set_error("mmasim_rms_norm: args is NULL"); return MMASIM_ERR_INVALID_ARG; }
    return run_rows("mmasim_rms_norm", fmt, M, K, *args, true, stream);
}

uint64_t mmasim_rms_norm_backward_workspace(int64_t M, int64_t K) {
    return M < 0 || M > 0x7FFFFFFF || K < 1 || K > ROWS_MAX_K ? 0 : rms_norm_backward_workspace(M, K);
}

int mmasim_rms_norm_backward(int fmt, int64_t M, int64_t K, const mmasim_rms_norm_backward_args* args, void* stream) {
    const char* call = "mmasim_rms_norm_backward";
    if (!args) { set_error("%s: args is NULL", call); return MMASIM_ERR_INVALID_ARG; }
    mmasim_rms_norm_backward_args p = *args;
    if (element_fmt(fmt) < 0) { set_error("%s: rows are FP32, BF16 or FP16", call); return MMASIM_ERR_INVALID_ARG; }
    if ((p.weight || p.dweight) && p.weight_fmt != fmt && p.weight_fmt != MMASIM_F32) { set_error("%s: the weight is of the rows' type or FP32", call); return MMASIM_ERR_INVALID_ARG; }
    if (!(p.eps >= 0.0f)) { set_error("%s: eps must be >= 0", call); return MMASIM_ERR_INVALID_ARG; }
    int st = check_shape(call, M, K, ROWS_MAX_K);
    if (st == MMASIM_OK) st = check_ld(call, "dy", &p.ld_dy, K);
    if (st == MMASIM_OK) st = check_ld(call, "h", &p.ld_h, K);
    if (st == MMASIM_OK) st = check_ld(call, "dresidual", &p.ld_dresidual, K);
    if (st == MMASIM_OK) st = check_ld(call, "dx", &p.ld_dx, K);
    if (st != MMASIM_OK) return st;
    if (M && (!p.dy || !p.h || !p.dx)) { set_error("%s: dy, h and dx must not be NULL", call); return MMASIM_ERR_INVALID_ARG; }
    if (!M) p.dy = p.h = p.dresidual = p.dx = nullptr;
    const uint64_t need = p.dweight ? rms_norm_backward_workspace(M, K) : 0;
    if (need && (!p.workspace || p.workspace_bytes < need)) {
        set_error("%s: dweight needs a workspace of %llu bytes", call, (unsigned long long)need);
        return MMASIM_ERR_INVALID_ARG;
    }
    if (!need) p.workspace = nullptr;
    const int b = element_bytes(fmt), wb = p.weight_fmt == MMASIM_F32 ? 4 : 2;
    const Span dy = {"dy", p.dy, M, K * b, p.ld_dy * b}, h = {"h", p.h, M, K * b, p.ld_h * b}, r = {"dresidual", p.dresidual, M, K * b, p.ld_dresidual * b},
               w = {"weight", p.weight, 1, K * wb, 0}, dx = {"dx", p.dx, M, K * b, p.ld_dx * b}, dw = {"dweight", p.dweight, 1, K * wb, 0},
               ws = {"workspace", p.workspace, 1, int64_t(need), 0};
    int device = 0;
    if ((st = current_device(call, &device)) != MMASIM_OK) return st;
    const Span* all[] = {&dy, &h, &r, &w, &dx, &dw, &ws};
    const int align[] = {b, b, b, wb, b, wb, 16};
    for (int i = 0; i < 7; ++i)
        if ((st = check_span(call, *all[i], align[i], device)) != MMASIM_OK) return st;
    for (int i = 4; i < 7; ++i)
        for (int j = 0; j < i; ++j) {
            const bool in_place = i == 4 && j < 3 && same_rows(*all[i], *all[j]);
            if (!in_place && meet(*all[i], *all[j])) { set_error("%s: %s lies over %s", call, all[i]->name, all[j]->name); return MMASIM_ERR_INVALID_ARG; }
        }
    return launch_rms_norm_backward(element_fmt(fmt), M, K, p, static_cast<cudaStream_t>(stream));
}

int mmasim_matvec4(int w_fmt, int fmt, int64_t T, int64_t N, int64_t K, const void* W, int64_t ldw, const void* sf, const float* row_scale,
                   const void* x, int64_t ldx, void* y, int64_t ldy, void* stream) {
    const char* call = "mmasim_matvec4";
    if (!packed4(w_fmt)) { set_error("%s: weights are MXF4_GST or NVF4_GST", call); return MMASIM_ERR_UNSUPPORTED; }
    if (element_fmt(fmt) < 0) { set_error("%s: x and y are FP32, BF16 or FP16", call); return MMASIM_ERR_INVALID_ARG; }
    if (T < 0 || T > 0x7FFFFFFF || N < 1 || N > 0x40000000 || K < 32 || K % 32 || K > (fmt == MMASIM_F32 ? MATVEC_MAX_K_F32 : ROWS_MAX_K)) {
        set_error("%s: T = %lld, N = %lld, K = %lld: T from 0 on, N from 1 to 2^30 and multiples of 32 up to %d (FP32: %d) for K are taken", call, (long long)T, (long long)N, (long long)K,
                  int(ROWS_MAX_K), int(MATVEC_MAX_K_F32));
        return MMASIM_ERR_SHAPE;
    }
    int st = check_ld(call, "W", &ldw, K);
    if (st == MMASIM_OK) st = check_ld(call, "x", &ldx, K);
    if (st == MMASIM_OK) st = check_ld(call, "y", &ldy, N);
    if (st != MMASIM_OK) return st;
    if (ldw % 32) { set_error("%s: the leading dimension of W must be a multiple of 32", call); return MMASIM_ERR_ALIGN; }
    if (T == 0) return MMASIM_OK;
    if (!W || !sf || !x || !y) { set_error("%s: W, sf, x and y must not be NULL", call); return MMASIM_ERR_INVALID_ARG; }
    const int b = element_bytes(fmt);
    const Span w = {"W", W, N, K / 2, ldw / 2}, s = {"sf", sf, 1, N * (K / block_of(w_fmt)), 0}, rs = {"row_scale", row_scale, 1, N * 4, 0},
               in = {"x", x, T, K * b, ldx * b}, out = {"y", y, T, N * b, ldy * b};
    int device = 0;
    if ((st = current_device(call, &device)) != MMASIM_OK) return st;
    const Span* all[] = {&w, &s, &rs, &in, &out};
    const int align[] = {16, w_fmt == MMASIM_NVF4_GST ? 2 : 1, 4, b, b};
    for (int i = 0; i < 5; ++i)
        if ((st = check_span(call, *all[i], align[i], device)) != MMASIM_OK) return st;
    for (int j = 0; j < 4; ++j)
        if (meet(out, *all[j])) { set_error("%s: y lies over %s", call, all[j]->name); return MMASIM_ERR_INVALID_ARG; }
    return launch_matvec4(w_fmt == MMASIM_NVF4_GST, element_fmt(fmt), T, N, K, W, ldw, sf, row_scale, x, ldx, y, ldy, static_cast<cudaStream_t>(stream));
}

}  // extern "C"
