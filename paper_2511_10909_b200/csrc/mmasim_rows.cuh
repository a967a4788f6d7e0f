// Rows into scaled operands: root-mean-square norm with the residual's addition (mmasim_rms_norm) and quantisation (mmasim_quantize), one
// kernel, one pass over the data.
//
//   h = x + residual, rounded to the rows' type and stored;  y = h / sqrt(mean h^2 + eps) * w in FP32;  y rounded once, or quantised:
//   row scales   s = max(max |y| / top, 2^-126), code = nearest(y / s)                                   E4M3, E5M2
//   blocks of 32 sf = floor(log2 max |y|) - emax (E8M0), code = nearest(y / 2^sf)                          MXE4M3, MXE5M2, MXF4
//   blocks of 16 s = max(row's max |y| / 2688, 2^-100), g = nearest UE4M3 of max |y| / 6s, code = nearest(y / gs)     NVF4
// with FP32 roundings in between: scales and quotients as plain FP32 arithmetic has them (Divisor), y as (h r) w with the mean from fl(1 / K), the
// sum of squares in the kernel's own order and r within 2^-23 (inverse_root).
//
// What bounds it is memory: 7 bytes an element for BF16 with a residual into FP8.  A row is `threads` threads (8, 16 or
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
    float eps, inverse_k;
    int e5m2;                               // FP8: which
    int w_f32;
    int vec_x, vec_r, vec_h, vec_o, vec_w;  // every row starts where eight elements can be moved at once
};

// Sum, or largest, of the row's threads, for all of them; `slot`: 16 words of shared memory that nothing else uses.
__device__ __forceinline__ float row_sum(float v, int threads, float* slot) {
    for (int o = min(threads, 32) / 2; o > 0; o >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, o);
    if (threads > 32) {
        if ((threadIdx.x & 31) == 0) slot[threadIdx.x >> 5] = v;
        __syncthreads();
        v = int(threadIdx.x & 15) < threads / 32 ? slot[threadIdx.x & 15] : 0.0f;
#pragma unroll
        for (int o = 8; o > 0; o >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, o);
    }
    return v;
}
__device__ __forceinline__ uint32_t row_max(uint32_t v, int threads, uint32_t* slot) {
    if (threads < 32) {
        for (int o = threads / 2; o > 0; o >>= 1) v = max(v, __shfl_xor_sync(0xFFFFFFFFu, v, o));
        return v;
    }
    v = __reduce_max_sync(0xFFFFFFFFu, v);
    if (threads > 32) {
        if ((threadIdx.x & 31) == 0) slot[threadIdx.x >> 5] = v;
        __syncthreads();
        v = __reduce_max_sync(0xFFFFFFFFu, int(threadIdx.x & 31) < threads / 32 ? slot[threadIdx.x & 31] : 0u);
    }
    return v;
}

template <int OUT, bool VEC> constexpr bool SPREAD_ROWS = !VEC && OUT != OUT_MXF4 && OUT != OUT_NVF4;

// VEC: rows of whole eights, all of which start on 16 bytes (codes: on their eight or four).  Other rows: an eight's elements lie a row's threads
// apart, neighbouring threads take neighbouring elements (a warp the 32 of a block); 4-bit codes, whose rows are whole blocks, as with VEC.
template <int T, int OUT, int V, bool NORM, bool VEC>
__global__ void __launch_bounds__(MAX_THREADS) rows_kernel(const Args a) {
    using namespace quant;
    using E = typename Elem<T>::type;
    __shared__ float sum_slot[16];
    __shared__ uint32_t max_slot[16];
    after_previous();
    const int per_cta = a.threads > 32 ? 1 : int(blockDim.x) / a.threads;
    const int64_t row = int64_t(blockIdx.x) * per_cta + (a.threads > 32 ? 0 : threadIdx.x / a.threads);
    const int t = a.threads > 32 ? threadIdx.x : threadIdx.x & (a.threads - 1);
    // NVF4: two eights side by side where a thread has several, one scale for both (BF16 4096 x 4096: 13.4 us without, 10.9 with; FP32 rows
    // read 64 bytes a thread that way, and a norm of 4096 x 4096 took 47 us, not 37)
    constexpr int SIDE = OUT == OUT_NVF4 && V > 1 && T != EF_F32 ? 2 : 1;
    constexpr bool SPREAD = SPREAD_ROWS<OUT, VEC>;
    auto place = [&](int j) { return SPREAD ? t + j * 8 * a.threads : (t + j / SIDE * a.threads) * (8 * SIDE) + j % SIDE * 8; };
    const int K = row < a.M ? a.K : 0;      // (threads of the last CTA without a row take part in the exchanges between lanes)
    const E* x = static_cast<const E*>(a.x) + row * a.ldx;

    Raw<T> h[V];
#pragma unroll
    for (int j = 0; j < V; ++j) {
        if constexpr (SPREAD) h[j] = load_spread<T>(x + place(j), K - place(j), a.threads);
        else h[j] = load8<T, VEC>(x + place(j), K - place(j), a.vec_x);
    }
    Pair y[NORM ? V : 1][4];                // without a norm the elements stay as they were loaded until their codes are made
    if constexpr (NORM) {
        if (a.residual) {
            const E* r = static_cast<const E*>(a.residual) + row * a.ldr;
            E* out = static_cast<E*>(a.h_out) + row * a.ldh;
            Raw<T> res[V];
#pragma unroll
            for (int j = 0; j < V; ++j) {
                if constexpr (SPREAD) res[j] = load_spread<T>(r + place(j), K - place(j), a.threads);
                else res[j] = load8<T, VEC>(r + place(j), K - place(j), a.vec_r);
            }
#pragma unroll
            for (int j = 0; j < V; ++j) {   // the norm is taken of what is stored: the backward pass has nothing else
                add_to<T>(h[j], res[j]);
                if constexpr (SPREAD) store_spread<T>(out + place(j), h[j], K - place(j), a.threads);
                else if (place(j) < K) store8<T, VEC>(out + place(j), h[j], K - place(j), a.vec_h);
            }
        }
        constexpr bool EARLY = V <= 2;      // asked for before the row's threads wait for one another, where the registers hold them
        Pair w[EARLY ? V : 1][4];
        auto weight = [&](int j, Pair (&to)[4]) {
            if constexpr (SPREAD) load_weight_spread<T>(a.w, a.w_f32, place(j), K - place(j), a.threads, to);
            else load_weight8<T, VEC>(a.w, a.w_f32, place(j), K - place(j), a.vec_w, to);
        };
#pragma unroll
        for (int j = 0; j < V && EARLY; ++j) weight(j, w[j]);
        Pair squares = 0;
#pragma unroll
        for (int j = 0; j < V; ++j) {
            widen<T>(h[j], y[j]);
#pragma unroll
            for (int i = 0; i < 4; ++i) squares = fma2(y[j][i], y[j][i], squares);
        }
        float even, odd;
        split(squares, even, odd);
        const Pair r = both(inverse_root(__fmaf_rn(row_sum(even + odd, a.threads, sum_slot), a.inverse_k, a.eps)));
        // (behind the row's end: zeros times zeros, and where r is not finite no element of the row is a number)
#pragma unroll
        for (int j = 0; j < V; ++j) {
            if constexpr (!EARLY) weight(j, w[0]);
#pragma unroll
            for (int i = 0; i < 4; ++i) y[j][i] = mul2(mul2(y[j][i], r), w[EARLY ? j : 0][i]);
        }
    }

    if constexpr (OUT == OUT_PLAIN) {
#pragma unroll
        for (int j = 0; j < V; ++j) {
            const int at = place(j);
            Raw<T> o;
            narrow<T>(y[j], o);
            if constexpr (SPREAD) store_spread<T>(static_cast<E*>(a.out) + row * a.ldo + at, o, K - at, a.threads);
            else if (at < K) store8<T, VEC>(static_cast<E*>(a.out) + row * a.ldo + at, o, K - at, a.vec_o);
        }
        return;
    }
    float scale = 0.0f, unit = 0.0f;        // of the row; NVF4: six times the scale
    if constexpr (OUT == OUT_FP8 || OUT == OUT_NVF4) {
        uint32_t top = 0u;
#pragma unroll
        for (int j = 0; j < V; ++j) {
            if constexpr (NORM) top = largest(top, y[j]);
            else largest_halves<T>(top, h[j]);
        }
        if constexpr (!NORM) top = largest_of<T>(top);
        top = row_max(top, a.threads, max_slot);
        if (top >= INF_BITS) scale = __uint_as_float(0x7FC00000u);
        else if constexpr (OUT == OUT_NVF4) scale = fmaxf(__fdiv_rn(__uint_as_float(top), 2688.0f), 7.88860905e-31f);       // 2^-100: g times it stays normal
        else scale = fmaxf(__fdiv_rn(__uint_as_float(top), a.e5m2 ? 57344.0f : 448.0f), 1.17549435e-38f);                    // 2^-126
        unit = __fmul_rn(6.0f, scale);
        if (t == 0 && K > 0) a.row_scale[row] = scale;
    }
    const Divisor by(OUT == OUT_NVF4 ? unit : scale);
#pragma unroll
    for (int j0 = 0; j0 < V; j0 += SIDE) {
        const int at = place(j0);
        Pair v[SIDE][4];
#pragma unroll
        for (int k = 0; k < SIDE; ++k) {
            if constexpr (!NORM) widen<T>(h[j0 + k], v[k]);
            else {
#pragma unroll
                for (int i = 0; i < 4; ++i) v[k][i] = y[j0 + k][i];
            }
        }
        bool zero = false;                  // FP4 has no code for a block without numbers
        if constexpr (OUT == OUT_FP8) by.apply(v[0]);
        if constexpr (SPREAD && OUT == OUT_MX8) {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                float lo, hi;
                split(v[0][i / 2], lo, hi);
                const int e = at + i * a.threads;
                const uint32_t code = e8m0_code(__reduce_max_sync(0xFFFFFFFFu, __float_as_uint(i & 1 ? hi : lo) & 0x7FFFFFFFu), a.e5m2 ? 15 : 8);
                v[0][i / 2] = i & 1 ? pair(lo, __fmul_rn(hi, e8m0_inverse(code))) : pair(__fmul_rn(lo, e8m0_inverse(code)), hi);
                if ((t & 31) == 0 && e < K) a.sf[row * a.ld_sf + e / 32] = uint8_t(code);
            }
        } else if constexpr (OUT == OUT_MX8 || OUT == OUT_MXF4) {
            uint32_t top = largest(0u, v[0]);
            top = max(top, __shfl_xor_sync(0xFFFFFFFFu, top, 1));
            top = max(top, __shfl_xor_sync(0xFFFFFFFFu, top, 2));
            const uint32_t code = e8m0_code(top, OUT == OUT_MXF4 ? 2 : (a.e5m2 ? 15 : 8));
            const Pair f = both(e8m0_inverse(code));
#pragma unroll
            for (int i = 0; i < 4; ++i) v[0][i] = mul2(v[0][i], f);
            zero = code == 255u;
            if ((t & 3) == 0 && at < K) a.sf[row * a.ld_sf + at / 32] = uint8_t(code);
        }
        if constexpr (OUT == OUT_NVF4) {
            uint32_t top = largest(0u, v[0]);
            if constexpr (SIDE == 2) top = largest(top, v[1]);
            else top = max(top, __shfl_xor_sync(0xFFFFFFFFu, top, 1));
            const uint32_t code = scale == scale ? ue4m3_code(by(__uint_as_float(top))) : 0x7Fu;
            const Divisor of(__fmul_rn(ue4m3_value(code), scale));
#pragma unroll
            for (int k = 0; k < SIDE; ++k) of.apply(v[k]);
            zero = code == 0x7Fu;
            if ((SIDE == 2 || (t & 1) == 0) && at < K) a.sf[row * a.ld_sf + at / 16] = uint8_t(code);
        }
        if (at >= K) continue;
        if constexpr (OUT == OUT_FP8 || OUT == OUT_MX8) {
            const uint2 c = a.e5m2 ? codes_e5m2(v[0]) : codes_e4m3(v[0]);
            uint8_t* p = static_cast<uint8_t*>(a.out) + row * a.ldo + at;
            if constexpr (VEC) *reinterpret_cast<uint2*>(p) = c;
            else {
#pragma unroll
                for (int i = 0; i < 8; ++i) if (at + i * a.threads < K) p[i * a.threads] = uint8_t((i < 4 ? c.x : c.y) >> (8 * (i & 3)));
            }
        } else {
            uint8_t* p = static_cast<uint8_t*>(a.out) + (row * a.ldo + at) / 2;
#pragma unroll
            for (int k = 0; k < SIDE; ++k, p += 4) {
                const uint32_t c = zero ? 0u : codes_e2m1(v[k]);
                if (VEC || a.vec_o) *reinterpret_cast<uint32_t*>(p) = c;     // (K is a multiple of 32)
                else {
#pragma unroll
                    for (int i = 0; i < 4; ++i) p[i] = uint8_t(c >> (8 * i));
                }
            }
        }
    }
}

// Threads per row and eights per thread.  Few rows are a matter of latency: the most threads.  Many rows are one of instructions, and what a
// thread does once a row (the exchanges, the scale) counts less with several eights; a row of a warp or less needs no barrier either, and a CTA
// then has several.  So, where all of a row's accesses are of 16 bytes, a row takes the fewest threads that still give every SM 512:
//   - with eight eights each where 16-bit rows are quantised with a scale of the row (us, threads per row before and now: E5M2 of 2048 x 14336
//     448 / 224, 20.7 / 15.7; E4M3 of 32768 x 512 64 / 8, 18.9 / 10.0; NVF4 of 4096 x 14336 448 / 224, 38.0 / 30.0);
//   - with four else, if the row is a warp's then: larger ones of CTAs of one or two warps gain nothing (MXFP8 of 32768 x 512 64 / 16, 18.6 / 9.3;
//     norm of 8192 x 2048 into E4M3 256 / 64, 24.8 / 21.7; of 65536 x 128 16 / 8, 8.6 / 6.9), nor do norms of FP32 rows (16384 x 512 64 / 16, 21 / 29).
// Others of many rows: a norm takes 256 threads, where its rows need more than four eights of them the fewest that do, quantisation 128.  BF16,
// 4096 x 4096, us with 512 / 256 / 128 threads: norm into MXFP8 23.5 / 21.1 / 22.2; norm of 16384 x 8192 into E4M3 with 512 / 256 threads 170 / 138.
constexpr int64_t FEW_ROWS = 296;
constexpr int SHORT_ROW = 256;              // eights
struct Shape { int threads, v; };
inline Shape shape(int64_t M, int K, bool norm, int most, bool whole_warps) {           // most: eights per thread where every access is of 16 bytes, else 1
    const int eights = (K + 7) / 8;
    int v = 1;
    if (M > FEW_ROWS && (most == 8 || eights <= SHORT_ROW))
        while (v < most && eights > v * 8 && M * eights >= 2 * v * 148 * 512) v *= 2;
    const int threads = (eights + v - 1) / v;
    if (threads <= 8 && !whole_warps) return {8, v};
    if (threads <= 16 && !whole_warps) return {16, v};
    if (threads <= 32) return {32, v};
    while (most < 8 && M > FEW_ROWS && v < 4 && eights > v * (norm ? 256 : 128)) v *= 2;
    while (eights > v * MAX_THREADS) v *= 2;
    return {((eights + v - 1) / v + 31) / 32 * 32, v};
}

template <int T, int OUT, bool NORM, bool VEC>
cudaError_t launch_out(const Args& a, int v, cudaStream_t stream) {
    const unsigned block = a.threads > 32 ? unsigned(a.threads) : 128u;
    const int per_cta = a.threads > 32 ? 1 : 128 / a.threads;
    const dim3 grid(unsigned((a.M + per_cta - 1) / per_cta));
    switch (v) {
        case 1: return enqueue(rows_kernel<T, OUT, 1, NORM, VEC>, grid, block, 0, stream, a);
        case 2: return enqueue(rows_kernel<T, OUT, 2, NORM, VEC>, grid, block, 0, stream, a);
        case 4: return enqueue(rows_kernel<T, OUT, 4, NORM, VEC>, grid, block, 0, stream, a);
        default: return enqueue(rows_kernel<T, OUT, 8, NORM, VEC>, grid, block, 0, stream, a);
    }
}
template <int T, int OUT>
cudaError_t launch_out(Args a, bool norm, cudaStream_t stream) {
    const bool vec = a.K % 8 == 0 && a.vec_x && a.vec_o && a.vec_w && (!a.residual || (a.vec_r && a.vec_h));
    constexpr bool ROW_SCALES = OUT == OUT_FP8 || OUT == OUT_NVF4;
    const int most = !vec || (norm && T == EF_F32) ? 1 : !norm && ROW_SCALES && T != EF_F32 ? 8 : 4;
    const Shape s = shape(a.M, a.K, norm, most, !vec && SPREAD_ROWS<OUT, false>);
    a.threads = s.threads;
    a.inverse_k = 1.0f / float(a.K);
    if constexpr (OUT != OUT_PLAIN)
        if (!norm) return vec ? launch_out<T, OUT, false, true>(a, s.v, stream) : launch_out<T, OUT, false, false>(a, s.v, stream);
    return vec ? launch_out<T, OUT, true, true>(a, s.v, stream) : launch_out<T, OUT, true, false>(a, s.v, stream);
}
template <int T>
cudaError_t launch_type(const Args& a, int out, bool norm, cudaStream_t stream) {
    switch (out) {
        case OUT_PLAIN: return launch_out<T, OUT_PLAIN>(a, norm, stream);
        case OUT_FP8: return launch_out<T, OUT_FP8>(a, norm, stream);
        case OUT_MX8: return launch_out<T, OUT_MX8>(a, norm, stream);
        case OUT_MXF4: return launch_out<T, OUT_MXF4>(a, norm, stream);
        default: return launch_out<T, OUT_NVF4>(a, norm, stream);
    }
}

// one per file: mmasim_rows_f32.cu, mmasim_rows_bf16.cu, mmasim_rows_f16.cu
cudaError_t launch_f32(const Args& a, int out, bool norm, cudaStream_t stream);
cudaError_t launch_bf16(const Args& a, int out, bool norm, cudaStream_t stream);
cudaError_t launch_f16(const Args& a, int out, bool norm, cudaStream_t stream);

}  // namespace rows
}  // namespace mmasim
