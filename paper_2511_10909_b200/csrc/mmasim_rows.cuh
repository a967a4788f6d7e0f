// Rows into scaled operands: root-mean-square norm with the residual's addition (mmasim_rms_norm) and quantisation (mmasim_quantize), one
// kernel, one pass over the data.
//
//   h = x + residual, rounded to the rows' type and stored;  y = h / sqrt(mean h^2 + eps) * w in FP32;  y rounded once, or quantised:
//   row scales   s = max(max |y| / top, 2^-126), code = nearest(y / s)                                   E4M3, E5M2
//   blocks of 32 sf = floor(log2 max |y|) - emax (E8M0), code = nearest(y / 2^sf)                          MXE4M3, MXE5M2, MXF4
//   blocks of 16 s = max(row's max |y| / 2688, 2^-100), g = nearest UE4M3 of max |y| / 6s, code = nearest(y / gs)     NVF4
// with FP32 roundings in between, as plain FP32 arithmetic has them (the sum of squares is the one value whose order is the kernel's own).
//
// What bounds it is memory: 7 bytes an element for BF16 with a residual into FP8, some 18 instructions.  A row is `threads` threads (8, 16 or
// 32 of a warp, or a CTA), each with V eights of consecutive elements `threads` eights apart, so that a warp's loads are contiguous and a
// block of 32 (16) is four (two) neighbouring lanes; the row stays in registers from the load to the codes.
#pragma once
#include "mmasim_quant.cuh"

namespace mmasim {
namespace rows {

enum Out : int { OUT_PLAIN = 0, OUT_FP8, OUT_MX8, OUT_MXF4, OUT_NVF4 };
constexpr int MAX_THREADS = 512;

struct Args {
    int64_t M;
    int K;
    int threads;                            // per row: 8, 16, 32, or blockDim.x
    const void *x, *residual, *w;
    void *h_out, *out;
    uint8_t* sf;
    float* row_scale;
    int64_t ldx, ldr, ldh, ldo, ld_sf;      // in elements (FP4: two per byte)
    float eps;
    int e5m2;                               // FP8: which
    int w_f32;
    int vec_x, vec_r, vec_h, vec_o, vec_w;  // every row starts where eight elements can be moved at once
};

// Sum, or largest, of the row's threads; `slot`: 16 words of shared memory that nothing else uses.
__device__ __forceinline__ float row_sum(float v, int threads, float* slot) {
    for (int o = min(threads, 32) / 2; o > 0; o >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, o);
    if (threads > 32) {
        if ((threadIdx.x & 31) == 0) slot[threadIdx.x >> 5] = v;
        __syncthreads();
        v = int(threadIdx.x & 31) < threads / 32 ? slot[threadIdx.x & 31] : 0.0f;
#pragma unroll
        for (int o = 8; o > 0; o >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, o);
    }
    return __shfl_sync(0xFFFFFFFFu, v, threads > 32 ? 0 : (threadIdx.x & 31) & ~(threads - 1));
}
__device__ __forceinline__ uint32_t row_max(uint32_t v, int threads, uint32_t* slot) {
    for (int o = min(threads, 32) / 2; o > 0; o >>= 1) v = max(v, __shfl_xor_sync(0xFFFFFFFFu, v, o));
    if (threads > 32) {
        if ((threadIdx.x & 31) == 0) slot[threadIdx.x >> 5] = v;
        __syncthreads();
        v = int(threadIdx.x & 31) < threads / 32 ? slot[threadIdx.x & 31] : 0u;
#pragma unroll
        for (int o = 8; o > 0; o >>= 1) v = max(v, __shfl_xor_sync(0xFFFFFFFFu, v, o));
        v = __shfl_sync(0xFFFFFFFFu, v, 0);
    }
    return v;
}

template <int T, int OUT, int V, bool NORM>
__global__ void __launch_bounds__(MAX_THREADS) rows_kernel(const Args a) {
    using namespace quant;
    using E = typename Elem<T>::type;
    __shared__ float sum_slot[16];
    __shared__ uint32_t max_slot[16];
    after_previous();
    const int per_cta = a.threads > 32 ? 1 : int(blockDim.x) / a.threads;
    const int64_t row = int64_t(blockIdx.x) * per_cta + (a.threads > 32 ? 0 : threadIdx.x / a.threads);
    const int t = a.threads > 32 ? threadIdx.x : threadIdx.x & (a.threads - 1);
    const bool live = row < a.M;            // (the others of the last CTA take part in the exchanges between lanes)
    const E* x = static_cast<const E*>(a.x) + row * a.ldx;

    float y[V][8];
    int n[V];                               // elements of this eight within the row
#pragma unroll
    for (int j = 0; j < V; ++j) {
        n[j] = live ? a.K - (t + j * a.threads) * 8 : 0;
        widen<T>(load8<T>(x + (n[j] > 0 ? (t + j * a.threads) * 8 : 0), n[j], a.vec_x), y[j]);
    }
    if constexpr (NORM) {
        if (a.residual) {
            const E* r = static_cast<const E*>(a.residual) + row * a.ldr;
            Raw<T> res[V];
#pragma unroll
            for (int j = 0; j < V; ++j) res[j] = load8<T>(r + (n[j] > 0 ? (t + j * a.threads) * 8 : 0), n[j], a.vec_r);
#pragma unroll
            for (int j = 0; j < V; ++j) {
                float v[8];
                widen<T>(res[j], v);
#pragma unroll
                for (int i = 0; i < 8; ++i) y[j][i] = __fadd_rn(y[j][i], v[i]);
                Raw<T> h;
                narrow<T>(y[j], h);
                widen<T>(h, y[j]);          // the norm is taken of what is stored: the backward pass has nothing else
                if (n[j] > 0) store8<T>(static_cast<E*>(a.h_out) + row * a.ldh + (t + j * a.threads) * 8, h, n[j], a.vec_h);
            }
        }
        float sum = 0.0f;
#pragma unroll
        for (int j = 0; j < V; ++j)
#pragma unroll
            for (int i = 0; i < 8; ++i) sum = __fmaf_rn(y[j][i], y[j][i], sum);
        const float r = __frsqrt_rn(__fadd_rn(__fdiv_rn(row_sum(sum, a.threads, sum_slot), float(a.K)), a.eps));
#pragma unroll
        for (int j = 0; j < V; ++j) {
            float w[8];
            load_weight8<T>(a.w, a.w_f32, n[j] > 0 ? (t + j * a.threads) * 8 : 0, n[j], a.vec_w, w);
#pragma unroll
            for (int i = 0; i < 8; ++i) y[j][i] = i < n[j] ? __fmul_rn(__fmul_rn(y[j][i], r), w[i]) : 0.0f;
        }
    }

    if constexpr (OUT == OUT_PLAIN) {
#pragma unroll
        for (int j = 0; j < V; ++j)
            if (n[j] > 0) {
                Raw<T> o;
                narrow<T>(y[j], o);
                store8<T>(static_cast<E*>(a.out) + row * a.ldo + (t + j * a.threads) * 8, o, n[j], a.vec_o);
            }
        return;
    }
    float scale = 0.0f;                     // of the row
    uint32_t amax[V];                       // of this eight, then of its block
#pragma unroll
    for (int j = 0; j < V; ++j) amax[j] = magnitude_bits(y[j]);
    if constexpr (OUT == OUT_FP8 || OUT == OUT_NVF4) {
        uint32_t top = 0u;
#pragma unroll
        for (int j = 0; j < V; ++j) top = max(top, amax[j]);
        top = row_max(top, a.threads, max_slot);
        if (top >= INF_BITS) scale = __uint_as_float(0x7FC00000u);
        else if constexpr (OUT == OUT_NVF4) scale = fmaxf(__fdiv_rn(__uint_as_float(top), 2688.0f), 7.88860905e-31f);       // 2^-100: g times it stays normal
        else scale = fmaxf(__fdiv_rn(__uint_as_float(top), a.e5m2 ? 57344.0f : 448.0f), 1.17549435e-38f);                    // 2^-126
        if (t == 0 && live) a.row_scale[row] = scale;
    }
    if constexpr (OUT == OUT_FP8) {
        const Divisor by(scale);
#pragma unroll
        for (int j = 0; j < V; ++j) by.apply(y[j]);
    }
#pragma unroll
    for (int j = 0; j < V; ++j) {
        const int at = (t + j * a.threads) * 8;
        bool zero = false;                  // FP4 has no code for a block without numbers
        if constexpr (OUT == OUT_MX8 || OUT == OUT_MXF4) {
            amax[j] = max(amax[j], __shfl_xor_sync(0xFFFFFFFFu, amax[j], 1));
            amax[j] = max(amax[j], __shfl_xor_sync(0xFFFFFFFFu, amax[j], 2));
            const uint32_t code = e8m0_code(amax[j], OUT == OUT_MXF4 ? 2 : (a.e5m2 ? 15 : 8));
            const float f = e8m0_inverse(code);
#pragma unroll
            for (int i = 0; i < 8; ++i) y[j][i] = __fmul_rn(y[j][i], f);
            zero = code == 255u;
            if ((t & 3) == 0 && n[j] > 0) a.sf[row * a.ld_sf + at / 32] = uint8_t(code);
        }
        if constexpr (OUT == OUT_NVF4) {
            amax[j] = max(amax[j], __shfl_xor_sync(0xFFFFFFFFu, amax[j], 1));
            const uint32_t code = scale == scale ? ue4m3_code(__fdiv_rn(__uint_as_float(amax[j]), __fmul_rn(6.0f, scale))) : 0x7Fu;
            Divisor(__fmul_rn(ue4m3_value(code), scale)).apply(y[j]);
            zero = code == 0x7Fu;
            if ((t & 1) == 0 && n[j] > 0) a.sf[row * a.ld_sf + at / 16] = uint8_t(code);
        }
        if (n[j] <= 0) continue;
        if constexpr (OUT == OUT_FP8 || OUT == OUT_MX8) {
            const uint2 c = a.e5m2 ? codes_e5m2(y[j]) : codes_e4m3(y[j]);
            uint8_t* p = static_cast<uint8_t*>(a.out) + row * a.ldo + at;
            if (a.vec_o && n[j] >= 8) *reinterpret_cast<uint2*>(p) = c;
            else {
#pragma unroll
                for (int i = 0; i < 8; ++i) if (i < n[j]) p[i] = uint8_t((i < 4 ? c.x : c.y) >> (8 * (i & 3)));
            }
        } else {
            const uint32_t c = zero ? 0u : codes_e2m1(y[j]);
            uint8_t* p = static_cast<uint8_t*>(a.out) + (row * a.ldo + at) / 2;
            if (a.vec_o) *reinterpret_cast<uint32_t*>(p) = c;                // (K is a multiple of 32)
            else {
#pragma unroll
                for (int i = 0; i < 4; ++i) p[i] = uint8_t(c >> (8 * i));
            }
        }
    }
}

// Threads per row and eights per thread.
struct Shape { int threads, v; };
inline Shape shape(int64_t M, int K) {
    const int eights = (K + 7) / 8;
    if (eights <= 8) return {8, 1};
    if (eights <= 16) return {16, 1};
    if (eights <= 32) return {32, 1};
    int v = 1;
    while (eights > v * MAX_THREADS) v *= 2;
    (void)M;
    return {((eights + v - 1) / v + 31) / 32 * 32, v};
}

template <int T, int OUT, bool NORM>
cudaError_t launch_out(const Args& a, int v, cudaStream_t stream) {
    const unsigned block = a.threads > 32 ? unsigned(a.threads) : 128u;
    const int per_cta = a.threads > 32 ? 1 : 128 / a.threads;
    const dim3 grid(unsigned((a.M + per_cta - 1) / per_cta));
    switch (v) {
        case 1: return enqueue(rows_kernel<T, OUT, 1, NORM>, grid, block, 0, stream, a);
        case 2: return enqueue(rows_kernel<T, OUT, 2, NORM>, grid, block, 0, stream, a);
        case 4: return enqueue(rows_kernel<T, OUT, 4, NORM>, grid, block, 0, stream, a);
        default: return enqueue(rows_kernel<T, OUT, 8, NORM>, grid, block, 0, stream, a);
    }
}
template <int T>
cudaError_t launch_type(Args a, int out, bool norm, cudaStream_t stream) {
    const Shape s = shape(a.M, a.K);
    a.threads = s.threads;
    switch (out) {
        case OUT_PLAIN: return launch_out<T, OUT_PLAIN, true>(a, s.v, stream);
        case OUT_FP8: return norm ? launch_out<T, OUT_FP8, true>(a, s.v, stream) : launch_out<T, OUT_FP8, false>(a, s.v, stream);
        case OUT_MX8: return norm ? launch_out<T, OUT_MX8, true>(a, s.v, stream) : launch_out<T, OUT_MX8, false>(a, s.v, stream);
        case OUT_MXF4: return norm ? launch_out<T, OUT_MXF4, true>(a, s.v, stream) : launch_out<T, OUT_MXF4, false>(a, s.v, stream);
        default: return norm ? launch_out<T, OUT_NVF4, true>(a, s.v, stream) : launch_out<T, OUT_NVF4, false>(a, s.v, stream);
    }
}

// one per file: mmasim_rows_f32.cu, mmasim_rows_bf16.cu, mmasim_rows_f16.cu
cudaError_t launch_f32(const Args& a, int out, bool norm, cudaStream_t stream);
cudaError_t launch_bf16(const Args& a, int out, bool norm, cudaStream_t stream);
cudaError_t launch_f16(const Args& a, int out, bool norm, cudaStream_t stream);

}  // namespace rows
}  // namespace mmasim
