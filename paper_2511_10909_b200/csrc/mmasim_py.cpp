// The call path of mmasim.gemm, mmasim.dot_batch and the operators on rows in native code: argument checks, output allocation, current
// stream, library call.  In Python these cost 13 us a call (probe batch of 2048 dots: 17.4 us with the launch), more than
// the kernels of small problems run.  Every function answers None when the call is not plain (anything but CUDA tensors of the expected
// types and strides, a status other than OK): the Python code then does it, and names what is wrong.
#include <torch/csrc/autograd/python_variable.h>
#include <ATen/ATen.h>
#include <ATen/cuda/EmptyTensor.h>
#include <c10/core/GradMode.h>
#include <c10/cuda/CUDAGuard.h>
#include <c10/cuda/CUDAStream.h>
#include "../../include/mmasim.h"

namespace {

decltype(&mmasim_gemm_ex) p_gemm_ex;
decltype(&mmasim_dot_batch) p_dot_batch;
decltype(&mmasim_model_info) p_model_info;
decltype(&mmasim_quantize) p_quantize;
decltype(&mmasim_rms_norm) p_rms_norm;
decltype(&mmasim_rms_norm_backward) p_rms_norm_backward;
decltype(&mmasim_rms_norm_backward_workspace) p_workspace;
decltype(&mmasim_matvec4) p_matvec4;

// bind(gemm_ex, dot_batch, model_info) and bind_rows(quantize, rms_norm, rms_norm_backward, its workspace, matvec4): addresses of the
// library's entry points.
bool addresses(PyObject* const* a, Py_ssize_t n, Py_ssize_t want, void** p) {
    if (n != want) { PyErr_Format(PyExc_TypeError, "%zd addresses are needed", want); return false; }
    for (Py_ssize_t i = 0; i < n; ++i) p[i] = PyLong_AsVoidPtr(a[i]);
    return !PyErr_Occurred();
}
PyObject* bind(PyObject*, PyObject* const* a, Py_ssize_t n) {
    void* p[3];
    if (!addresses(a, n, 3, p)) return nullptr;
    p_gemm_ex = reinterpret_cast<decltype(p_gemm_ex)>(p[0]);
    p_dot_batch = reinterpret_cast<decltype(p_dot_batch)>(p[1]);
    p_model_info = reinterpret_cast<decltype(p_model_info)>(p[2]);
    Py_RETURN_NONE;
}
PyObject* bind_rows(PyObject*, PyObject* const* a, Py_ssize_t n) {
    void* p[5];
    if (!addresses(a, n, 5, p)) return nullptr;
    p_quantize = reinterpret_cast<decltype(p_quantize)>(p[0]);
    p_rms_norm = reinterpret_cast<decltype(p_rms_norm)>(p[1]);
    p_rms_norm_backward = reinterpret_cast<decltype(p_rms_norm_backward)>(p[2]);
    p_workspace = reinterpret_cast<decltype(p_workspace)>(p[3]);
    p_matvec4 = reinterpret_cast<decltype(p_matvec4)>(p[4]);
    Py_RETURN_NONE;
}

const at::Tensor* tensor(PyObject* o) {                 // a plain CUDA tensor, or nothing
    if (!THPVariable_CheckExact(o)) return nullptr;
    const at::Tensor& t = THPVariable_Unpack(o);
    return t.defined() && t.layout() == at::kStrided && t.is_cuda() ? &t : nullptr;
}
// Row stride of a matrix of at least rows x cols words of `bytes` bytes on `dev`, or -1.
int64_t matrix(const at::Tensor* t, int64_t rows, int64_t cols, int bytes, at::Device dev) {
    if (!t || t->device() != dev || t->itemsize() != bytes || t->dim() != 2 || t->size(0) < rows || t->size(1) < cols) return -1;
    if (t->size(1) > 1 && t->stride(1) != 1) return -1;
    const int64_t ld = t->size(0) > 1 ? t->stride(0) : std::max(t->stride(0), t->size(1));
    return ld < cols ? -1 : ld;
}
bool vector(const at::Tensor* t, int64_t n, int bytes, at::Device dev) {
    return t && t->device() == dev && t->is_contiguous() && t->itemsize() == bytes && t->numel() >= n;
}
at::ScalarType word(int bytes) { return bytes == 8 ? at::kLong : (bytes == 4 ? at::kInt : at::kShort); }
void* stream() { return c10::cuda::getCurrentCUDAStream().stream(); }

// gemm(model, A, B, C, out, K, sfa, sfb, k_chunk, row_scale, col_scale, flags) -> D or None
PyObject* gemm(PyObject*, PyObject* const* a, Py_ssize_t n) {
    if (n != 12) Py_RETURN_NONE;
    const auto* model = static_cast<const mmasim_model*>(PyLong_AsVoidPtr(a[0]));
    mmasim_info info;
    if (PyErr_Occurred() || !model || p_model_info(model, &info)) { PyErr_Clear(); Py_RETURN_NONE; }
    const at::Tensor *A = tensor(a[1]), *B = tensor(a[2]);
    if (!A || !B || A->dim() != 2 || B->dim() != 2) Py_RETURN_NONE;
    const at::Device dev = A->device();
    const int64_t per_word = info.a_bits == 4 ? 2 : 1, M = A->size(0), N = B->size(0);
    const int64_t K = a[5] == Py_None ? A->size(1) * per_word : PyLong_AsLongLong(a[5]);
    const int64_t k_chunk = PyLong_AsLongLong(a[8]);
    const long flags = PyLong_AsLong(a[11]);
    if (PyErr_Occurred()) { PyErr_Clear(); Py_RETURN_NONE; }
    const int64_t words = (K + per_word - 1) / per_word, ld_a = matrix(A, M, words, std::max(info.a_bits, 8) / 8, dev),
                  ld_b = matrix(B, N, words, std::max(info.b_bits, 8) / 8, dev);
    if (K < 1 || ld_a < 0 || ld_b < 0) Py_RETURN_NONE;
    mmasim_gemm_opts o = {};
    o.lda = ld_a * per_word;
    o.ldb = ld_b * per_word;
    o.k_chunk = k_chunk;
    o.flags = int32_t(flags);
    const at::Tensor* C = nullptr;
    if (a[3] != Py_None) {
        C = tensor(a[3]);
        if ((o.ldc = matrix(C, M, N, info.acc_bytes, dev)) < 0) Py_RETURN_NONE;
    }
    if (info.k_block) {
        const int64_t nsf = (K + info.k_block - 1) / info.k_block;
        const at::Tensor *sa = tensor(a[6]), *sb = tensor(a[7]);
        if (matrix(sa, M, nsf, 1, dev) != nsf || matrix(sb, N, nsf, 1, dev) != nsf) Py_RETURN_NONE;
        o.sfa = sa->data_ptr();
        o.sfb = sb->data_ptr();
    } else if (a[6] != Py_None || a[7] != Py_None) Py_RETURN_NONE;
    if (a[9] != Py_None || a[10] != Py_None) {
        const at::Tensor *rs = tensor(a[9]), *cs = tensor(a[10]);
        if (!vector(rs, M, 4, dev) || !vector(cs, N, 4, dev)) Py_RETURN_NONE;
        o.row_scale = static_cast<const float*>(rs->data_ptr());
        o.col_scale = static_cast<const float*>(cs->data_ptr());
    }
    try {
        at::Tensor fresh;
        const at::Tensor* out = &fresh;
        if (a[4] == Py_None) fresh = at::empty({M, N}, at::TensorOptions().dtype(word(info.acc_bytes)).device(dev));
        else out = tensor(a[4]);
        if ((o.ldd = matrix(out, M, N, info.acc_bytes, dev)) < 0) Py_RETURN_NONE;
        const void *a_ptr = A->data_ptr(), *b_ptr = B->data_ptr(), *c_ptr = C ? C->data_ptr() : nullptr;
        void *d_ptr = out->data_ptr(), *s = stream();
        int st;
        Py_BEGIN_ALLOW_THREADS                              // (a launch waits where the stream's queue is full, an allocation too)
        st = p_gemm_ex(model, M, N, K, a_ptr, b_ptr, c_ptr, d_ptr, &o, s);
        Py_END_ALLOW_THREADS
        if (st) Py_RETURN_NONE;
        if (a[4] == Py_None) return THPVariable_Wrap(fresh);
        Py_INCREF(a[4]);
        return a[4];
    } catch (const std::exception&) { Py_RETURN_NONE; }
}

// dot_batch(model, A, B, C, out) -> D or None
PyObject* dot_batch(PyObject*, PyObject* const* a, Py_ssize_t n) {
    if (n != 5) Py_RETURN_NONE;
    const auto* model = static_cast<const mmasim_model*>(PyLong_AsVoidPtr(a[0]));
    mmasim_info info;
    if (PyErr_Occurred() || !model || p_model_info(model, &info)) { PyErr_Clear(); Py_RETURN_NONE; }
    const at::Tensor *A = tensor(a[1]), *B = tensor(a[2]), *C = a[3] == Py_None ? nullptr : tensor(a[3]);
    if (!A || A->dim() != 2 || (a[3] != Py_None && !C)) Py_RETURN_NONE;
    const at::Device dev = A->device();
    const int64_t dots = A->size(0), K = A->size(1);
    const int64_t ld_a = matrix(A, dots, K, std::max(info.a_bits, 8) / 8, dev), ld_b = matrix(B, dots, K, std::max(info.b_bits, 8) / 8, dev);
    if (K < 1 || ld_a < 0 || ld_b < 0 || (dots > 1 && (ld_a != K || ld_b != K))) Py_RETURN_NONE;
    if (C && !vector(C, dots, info.acc_bytes, dev)) Py_RETURN_NONE;
    try {
        at::Tensor fresh;
        const at::Tensor* out = &fresh;
        if (a[4] == Py_None) fresh = at::empty({dots}, at::TensorOptions().dtype(word(info.acc_bytes)).device(dev));
        else out = tensor(a[4]);
        if (!vector(out, dots, info.acc_bytes, dev)) Py_RETURN_NONE;
        const void *a_ptr = A->data_ptr(), *b_ptr = B->data_ptr(), *c_ptr = C ? C->data_ptr() : nullptr;
        void *d_ptr = out->data_ptr(), *s = stream();
        int st;
        Py_BEGIN_ALLOW_THREADS
        st = p_dot_batch(model, dots, K, a_ptr, b_ptr, c_ptr, d_ptr, s);
        Py_END_ALLOW_THREADS
        if (st) Py_RETURN_NONE;
        if (a[4] == Py_None) return THPVariable_Wrap(fresh);
        Py_INCREF(a[4]);
        return a[4];
    } catch (const std::exception&) { Py_RETURN_NONE; }
}

// ---- the operators on rows ----
// A new tensor straight from the allocator: by way of the dispatcher one takes 1.1 us, not 0.8 (with its end), and a norm into FP8 makes three.
at::Tensor empty(at::IntArrayRef shape, at::ScalarType type, at::Device dev) { return at::Tensor(at::detail::empty_cuda(shape, type, dev, std::nullopt)); }
int row_fmt(const at::Tensor& t) {
    const at::ScalarType s = t.scalar_type();
    return s == at::kFloat ? MMASIM_F32 : s == at::kBFloat16 ? MMASIM_BF16 : s == at::kHalf ? MMASIM_F16 : -1;
}
// Leading dimension of a rows x cols matrix of `type` on `dev`, or -1.
int64_t rows_ld(const at::Tensor* t, int64_t rows, int64_t cols, at::ScalarType type, at::Device dev) {
    if (!t || t->device() != dev || t->scalar_type() != type || t->dim() != 2 || t->size(0) != rows || t->size(1) != cols) return -1;
    if (cols > 1 && t->stride(1) != 1 && t->numel()) return -1;
    if (rows <= 1) return cols;
    return t->stride(0) < cols ? -1 : t->stride(0);
}
bool packed(const at::Tensor* t, at::IntArrayRef shape, at::ScalarType type, at::Device dev) {
    return t && t->device() == dev && t->scalar_type() == type && t->sizes() == shape && t->is_contiguous();
}
bool given(PyObject* o, const at::Tensor** t) {         // false: something else than None or a CUDA tensor
    *t = o == Py_None ? nullptr : tensor(o);
    return o == Py_None || *t;
}
// Autograd would be asked for a gradient through it, and no call records one.
bool traced(const at::Tensor* t) { return t && t->requires_grad() && c10::GradMode::is_enabled(); }
PyObject* result(PyObject* given_one, const at::Tensor& fresh, bool any) {      // a new reference
    if (given_one != Py_None) { Py_INCREF(given_one); return given_one; }
    if (any) return THPVariable_Wrap(fresh);
    Py_RETURN_NONE;
}
// Codes, sf and row_scale of a quantised matrix: the caller's (a[0..2], None = new ones).
struct Codes {
    int fmt;
    int64_t block = 0, per_byte = 1, ld = 0;
    bool row_scaled = false;
    at::Tensor fresh[3];
    const at::Tensor* t[3] = {nullptr, nullptr, nullptr};

    bool take(int f, PyObject* const* a, int64_t M, int64_t K, at::Device dev) {
        fmt = f;
        block = f == MMASIM_NVF4_GST ? 16 : (f == MMASIM_MXE4M3 || f == MMASIM_MXE5M2 || f == MMASIM_MXF4_GST ? 32 : 0);
        row_scaled = f == MMASIM_E4M3 || f == MMASIM_E5M2 || f == MMASIM_NVF4_GST;
        if (!block && !row_scaled) return false;
        per_byte = f == MMASIM_MXF4_GST || f == MMASIM_NVF4_GST ? 2 : 1;
        if (K < 1 || (per_byte == 2 && K % 32)) return false;
        const bool want[3] = {true, block != 0, row_scaled};
        for (int i = 0; i < 3; ++i) {
            if (!given(a[i], &t[i]) || (t[i] && !want[i]) || (a[0] != Py_None && want[i] && !t[i]) || (a[0] == Py_None && t[i])) return false;
        }
        if (!t[0]) {
            fresh[0] = empty({M, K / per_byte}, at::kByte, dev);
            if (want[1]) fresh[1] = empty({M, (K + block - 1) / block}, at::kByte, dev);
            if (want[2]) fresh[2] = empty({M}, at::kFloat, dev);
            for (int i = 0; i < 3; ++i) if (want[i]) t[i] = &fresh[i];
        }
        ld = rows_ld(t[0], M, K / per_byte, at::kByte, dev) * per_byte;
        return ld > 0 && (!want[1] || packed(t[1], {M, (K + block - 1) / block}, at::kByte, dev)) && (!want[2] || packed(t[2], {M}, at::kFloat, dev));
    }
    void* sf() const { return t[1] ? t[1]->data_ptr() : nullptr; }
    float* row_scale() const { return t[2] ? static_cast<float*>(t[2]->data_ptr()) : nullptr; }
};
bool weight_of(PyObject* o, int64_t K, const at::Tensor& x, int x_fmt, const at::Tensor** w, int* fmt) {
    if (!given(o, w)) return false;
    *fmt = x_fmt;
    if (!*w) return true;
    if ((*w)->scalar_type() == at::kFloat) *fmt = MMASIM_F32;
    else if ((*w)->scalar_type() != x.scalar_type()) return false;
    return packed(*w, {K}, (*w)->scalar_type(), x.device());
}

// quantize(x, fmt, codes, sf, row_scale) -> (codes, sf, row_scale) or None
PyObject* quantize(PyObject*, PyObject* const* a, Py_ssize_t n) {
    if (n != 5) Py_RETURN_NONE;
    const at::Tensor* x = tensor(a[0]);
    const long fmt = PyLong_AsLong(a[1]);
    if (PyErr_Occurred()) { PyErr_Clear(); Py_RETURN_NONE; }
    if (!x || x->dim() != 2) Py_RETURN_NONE;
    const at::Device dev = x->device();
    const int64_t M = x->size(0), K = x->size(1), ldx = rows_ld(x, M, K, x->scalar_type(), dev);
    const int in = row_fmt(*x);
    if (in < 0 || ldx < 1) Py_RETURN_NONE;
    try {
        const c10::cuda::OptionalCUDAGuard guard(dev);
        Codes c;
        if (!c.take(int(fmt), a + 2, M, K, dev)) Py_RETURN_NONE;
        const void* p = x->data_ptr();
        void *codes = c.t[0]->data_ptr(), *s = stream();
        int st;
        Py_BEGIN_ALLOW_THREADS
        st = p_quantize(in, int(fmt), M, K, p, ldx, codes, c.ld, c.sf(), c.row_scale(), s);
        Py_END_ALLOW_THREADS
        if (st) Py_RETURN_NONE;
        PyObject* r = PyTuple_New(3);
        for (int i = 0; r && i < 3; ++i) PyTuple_SET_ITEM(r, i, result(a[2 + i], c.fresh[i], c.fresh[i].defined()));
        return r;
    } catch (const std::exception&) { Py_RETURN_NONE; }
}

// rms_norm(x, weight, residual, eps, fmt, residual_out, out or codes, sf, row_scale) -> (out or codes, sf, row_scale, residual_out) or None; fmt -2: plain
PyObject* rms_norm(PyObject*, PyObject* const* a, Py_ssize_t n) {
    if (n != 9) Py_RETURN_NONE;
    const at::Tensor *x = tensor(a[0]), *w, *res, *res_out, *out;
    const double eps = PyFloat_AsDouble(a[3]);
    const long fmt = PyLong_AsLong(a[4]);
    if (PyErr_Occurred()) { PyErr_Clear(); Py_RETURN_NONE; }
    if (!x || x->dim() != 2 || !given(a[2], &res) || !given(a[5], &res_out) || !given(a[6], &out) || (res_out && !res)) Py_RETURN_NONE;
    const at::Device dev = x->device();
    const at::ScalarType type = x->scalar_type();
    const int64_t M = x->size(0), K = x->size(1);
    mmasim_rms_norm_args p = {};
    const int in = row_fmt(*x);
    if (in < 0 || K < 1 || (p.ldx = rows_ld(x, M, K, type, dev)) < 1 || !weight_of(a[1], K, *x, in, &w, &p.weight_fmt)) Py_RETURN_NONE;
    if ((fmt == -2 || res) && (traced(x) || traced(res) || (fmt == -2 && traced(w)))) Py_RETURN_NONE;
    try {
        const c10::cuda::OptionalCUDAGuard guard(dev);
        at::Tensor fresh_out, fresh_res;
        Codes c;
        if (res) {
            if (!res_out) { fresh_res = empty({M, K}, type, dev); res_out = &fresh_res; }
            if ((p.ld_residual = rows_ld(res, M, K, type, dev)) < 1 || (p.ld_residual_out = rows_ld(res_out, M, K, type, dev)) < 1) Py_RETURN_NONE;
            p.residual = res->data_ptr();
            p.residual_out = res_out->data_ptr();
        }
        if (fmt == -2) {
            if (!out) { fresh_out = empty({M, K}, type, dev); out = &fresh_out; }
            if ((p.ld_out = rows_ld(out, M, K, type, dev)) < 1) Py_RETURN_NONE;
            p.out = out->data_ptr();
            p.out_fmt = in;
        } else {
            if (!c.take(int(fmt), a + 6, M, K, dev)) Py_RETURN_NONE;
            p.out = c.t[0]->data_ptr();
            p.ld_out = c.ld;
            p.sf = c.sf();
            p.row_scale = c.row_scale();
            p.out_fmt = int(fmt);
        }
        p.x = x->data_ptr();
        p.weight = w ? w->data_ptr() : nullptr;
        p.eps = float(eps);
        void* s = stream();
        int st;
        Py_BEGIN_ALLOW_THREADS
        st = p_rms_norm(in, M, K, &p, s);
        Py_END_ALLOW_THREADS
        if (st) Py_RETURN_NONE;
        PyObject* r = PyTuple_New(4);
        if (!r) return nullptr;
        for (int i = 0; i < 3; ++i) {
            const at::Tensor& f = fmt == -2 && i == 0 ? fresh_out : c.fresh[i];
            PyTuple_SET_ITEM(r, i, result(a[6 + i], f, f.defined()));
        }
        PyTuple_SET_ITEM(r, 3, result(a[5], fresh_res, fresh_res.defined()));
        return r;
    } catch (const std::exception&) { Py_RETURN_NONE; }
}

// rms_norm_backward(dy, h, weight, dresidual, eps, need_dweight, dx) -> (dx, dweight) or None
PyObject* rms_norm_backward(PyObject*, PyObject* const* a, Py_ssize_t n) {
    if (n != 7) Py_RETURN_NONE;
    const at::Tensor *dy = tensor(a[0]), *h = tensor(a[1]), *w, *res, *dx;
    const double eps = PyFloat_AsDouble(a[4]);
    if (PyErr_Occurred()) { PyErr_Clear(); Py_RETURN_NONE; }
    const int need = PyObject_IsTrue(a[5]);
    if (need < 0) { PyErr_Clear(); Py_RETURN_NONE; }
    if (!dy || !h || h->dim() != 2 || !given(a[3], &res) || !given(a[6], &dx)) Py_RETURN_NONE;
    const at::Device dev = h->device();
    const at::ScalarType type = h->scalar_type();
    const int64_t M = h->size(0), K = h->size(1);
    mmasim_rms_norm_backward_args p = {};
    const int in = row_fmt(*h);
    if (in < 0 || K < 1 || (p.ld_h = rows_ld(h, M, K, type, dev)) < 1 || (p.ld_dy = rows_ld(dy, M, K, type, dev)) < 1 || !weight_of(a[2], K, *h, in, &w, &p.weight_fmt)
        || (res && (p.ld_dresidual = rows_ld(res, M, K, type, dev)) < 1)) Py_RETURN_NONE;
    try {
        const c10::cuda::OptionalCUDAGuard guard(dev);
        at::Tensor fresh_dx, dweight, workspace;
        if (!dx) { fresh_dx = empty({M, K}, type, dev); dx = &fresh_dx; }
        if ((p.ld_dx = rows_ld(dx, M, K, type, dev)) < 1) Py_RETURN_NONE;
        if (need) {
            dweight = empty({K}, w ? w->scalar_type() : type, dev);
            p.workspace_bytes = p_workspace(M, K);
            workspace = empty({int64_t(p.workspace_bytes)}, at::kByte, dev);
            p.dweight = dweight.data_ptr();
            p.workspace = workspace.data_ptr();
        }
        p.dy = dy->data_ptr();
        p.h = h->data_ptr();
        p.weight = w ? w->data_ptr() : nullptr;
        p.dresidual = res ? res->data_ptr() : nullptr;
        p.dx = dx->data_ptr();
        p.eps = float(eps);
        void* s = stream();
        int st;
        Py_BEGIN_ALLOW_THREADS
        st = p_rms_norm_backward(in, M, K, &p, s);
        Py_END_ALLOW_THREADS
        if (st) Py_RETURN_NONE;
        PyObject* r = PyTuple_New(2);
        if (!r) return nullptr;
        PyTuple_SET_ITEM(r, 0, result(a[6], fresh_dx, true));
        PyTuple_SET_ITEM(r, 1, result(Py_None, dweight, dweight.defined()));
        return r;
    } catch (const std::exception&) { Py_RETURN_NONE; }
}

// matvec4(fmt, W, sf, x, row_scale, out) -> y or None
PyObject* matvec4(PyObject*, PyObject* const* a, Py_ssize_t n) {
    if (n != 6) Py_RETURN_NONE;
    const long fmt = PyLong_AsLong(a[0]);
    if (PyErr_Occurred()) { PyErr_Clear(); Py_RETURN_NONE; }
    const at::Tensor *W = tensor(a[1]), *sf = tensor(a[2]), *x = tensor(a[3]), *rs, *out;
    if (!W || !sf || !x || W->dim() != 2 || x->dim() != 2 || !given(a[4], &rs) || !given(a[5], &out) || (fmt != MMASIM_MXF4_GST && fmt != MMASIM_NVF4_GST)) Py_RETURN_NONE;
    const at::Device dev = x->device();
    const int64_t T = x->size(0), K = x->size(1), N = W->size(0), block = fmt == MMASIM_NVF4_GST ? 16 : 32;
    const int in = row_fmt(*x);
    if (in < 0 || K < 1 || K % 32 || N < 1) Py_RETURN_NONE;
    const int64_t ldx = rows_ld(x, T, K, x->scalar_type(), dev), ldw = rows_ld(W, N, K / 2, at::kByte, dev) * 2;
    if (ldx < 1 || ldw < 1 || !packed(sf, {N, K / block}, at::kByte, dev) || (rs && !packed(rs, {N}, at::kFloat, dev))) Py_RETURN_NONE;
    if (traced(x) || traced(rs)) Py_RETURN_NONE;
    try {
        const c10::cuda::OptionalCUDAGuard guard(dev);
        at::Tensor fresh;
        if (!out) { fresh = empty({T, N}, x->scalar_type(), dev); out = &fresh; }
        const int64_t ldy = rows_ld(out, T, N, x->scalar_type(), dev);
        if (ldy < 1) Py_RETURN_NONE;
        const void *w = W->data_ptr(), *s_ptr = sf->data_ptr(), *x_ptr = x->data_ptr();
        const float* scale = rs ? static_cast<const float*>(rs->data_ptr()) : nullptr;
        void *y = out->data_ptr(), *s = stream();
        int st;
        Py_BEGIN_ALLOW_THREADS
        st = p_matvec4(int(fmt), in, T, N, K, w, ldw, s_ptr, scale, x_ptr, ldx, y, ldy, s);
        Py_END_ALLOW_THREADS
        if (st) Py_RETURN_NONE;
        return result(a[5], fresh, true);
    } catch (const std::exception&) { Py_RETURN_NONE; }
}

PyMethodDef methods[] = {
    {"bind", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(bind)), METH_FASTCALL, nullptr},
    {"bind_rows", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(bind_rows)), METH_FASTCALL, nullptr},
    {"gemm", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(gemm)), METH_FASTCALL, nullptr},
    {"dot_batch", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(dot_batch)), METH_FASTCALL, nullptr},
    {"quantize", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(quantize)), METH_FASTCALL, nullptr},
    {"rms_norm", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(rms_norm)), METH_FASTCALL, nullptr},
    {"rms_norm_backward", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(rms_norm_backward)), METH_FASTCALL, nullptr},
    {"matvec4", reinterpret_cast<PyCFunction>(reinterpret_cast<void*>(matvec4)), METH_FASTCALL, nullptr},
    {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_mmasim_py", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__mmasim_py() {
    PyObject* m = PyModule_Create(&module);
    if (m && PyModule_AddStringConstant(m, "built_against", MMASIM_BUILT_AGAINST)) { Py_DECREF(m); return nullptr; }
    return m;
}
