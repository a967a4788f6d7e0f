// Scaled 8- and 4-bit operands made on the GPU: scale factors from largest magnitudes, codes, and the element types that rows come in.
// Shared by mmasim_quantize, mmasim_rms_norm and mmasim_matvec4.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include "mmasim_internal.h"

namespace mmasim {
namespace quant {

constexpr uint32_t INF_BITS = 0x7F800000u;

// ---- eight consecutive elements of a row: as loaded (Raw) and as FP32 ----
template <int T> struct Elem;
template <> struct Elem<EF_F32> { using type = float; static constexpr int WORDS = 8; };
template <> struct Elem<EF_BF16> { using type = __nv_bfloat16; static constexpr int WORDS = 4; };
template <> struct Elem<EF_F16> { using type = __half; static constexpr int WORDS = 4; };
template <int T> struct Raw { uint32_t w[Elem<T>::WORDS]; };

template <int T> __device__ __forceinline__ void widen(const Raw<T>& r, float (&v)[8]) {
    if constexpr (T == EF_F32) {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = __uint_as_float(r.w[i]);
    } else if constexpr (T == EF_BF16) {
#pragma unroll
        for (int i = 0; i < 4; ++i) { v[2 * i] = __uint_as_float(r.w[i] << 16); v[2 * i + 1] = __uint_as_float(r.w[i] & 0xFFFF0000u); }
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&r.w[i]));
            v[2 * i] = f.x;
            v[2 * i + 1] = f.y;
        }
    }
}
template <int T> __device__ __forceinline__ void narrow(const float (&v)[8], Raw<T>& r) {       // to nearest, once
    if constexpr (T == EF_F32) {
#pragma unroll
        for (int i = 0; i < 8; ++i) r.w[i] = __float_as_uint(v[i]);
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if constexpr (T == EF_BF16) asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r.w[i]) : "f"(v[2 * i + 1]), "f"(v[2 * i]));
            else asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r.w[i]) : "f"(v[2 * i + 1]), "f"(v[2 * i]));
        }
    }
}
// The first `n` of eight elements (the rest zeros).  `vec`: the address is a multiple of 16 bytes.
template <int T> __device__ __forceinline__ Raw<T> load8(const typename Elem<T>::type* p, int n, bool vec) {
    Raw<T> r;
    if (vec && n >= 8) {
#pragma unroll
        for (int i = 0; i < Elem<T>::WORDS; i += 4) {
            const uint4 q = reinterpret_cast<const uint4*>(p)[i / 4];
            r.w[i] = q.x; r.w[i + 1] = q.y; r.w[i + 2] = q.z; r.w[i + 3] = q.w;
        }
    } else if constexpr (T == EF_F32) {
#pragma unroll
        for (int i = 0; i < 8; ++i) r.w[i] = i < n ? __float_as_uint(p[i]) : 0u;
    } else {
        const unsigned short* s = reinterpret_cast<const unsigned short*>(p);
#pragma unroll
        for (int i = 0; i < 4; ++i) r.w[i] = (2 * i < n ? uint32_t(s[2 * i]) : 0u) | (2 * i + 1 < n ? uint32_t(s[2 * i + 1]) << 16 : 0u);
    }
    return r;
}
template <int T> __device__ __forceinline__ void store8(typename Elem<T>::type* p, const Raw<T>& r, int n, bool vec) {
    if (vec && n >= 8) {
#pragma unroll
        for (int i = 0; i < Elem<T>::WORDS; i += 4) reinterpret_cast<uint4*>(p)[i / 4] = make_uint4(r.w[i], r.w[i + 1], r.w[i + 2], r.w[i + 3]);
    } else if constexpr (T == EF_F32) {
#pragma unroll
        for (int i = 0; i < 8; ++i) if (i < n) p[i] = __uint_as_float(r.w[i]);
    } else {
        unsigned short* s = reinterpret_cast<unsigned short*>(p);
#pragma unroll
        for (int i = 0; i < 8; ++i) if (i < n) s[i] = (unsigned short)(i & 1 ? r.w[i / 2] >> 16 : r.w[i / 2]);
    }
}
// Eight weights of a norm: of the rows' type or FP32, or ones.
template <int T> __device__ __forceinline__ void load_weight8(const void* w, bool f32, int at, int n, bool vec, float (&v)[8]) {
    if (!w) {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = 1.0f;
    } else if (f32) widen<EF_F32>(load8<EF_F32>(static_cast<const float*>(w) + at, n, vec), v);
    else widen<T>(load8<T>(static_cast<const typename Elem<T>::type*>(w) + at, n, vec), v);
}

// ---- codes ----
__device__ __forceinline__ uint32_t magnitude_bits(const float (&v)[8]) {       // (as integers NaN > infinity > finite magnitudes)
    uint32_t m = 0u;
#pragma unroll
    for (int i = 0; i < 8; ++i) m = max(m, __float_as_uint(v[i]) & 0x7FFFFFFFu);
    return m;
}
// q = x / t rounded to nearest, r = 1 / t: the product with the reciprocal, corrected twice by its exact remainder (Markstein, Computation of
// elementary functions on the IBM RISC System/6000, 1990).  The remainder is exact, and t's reciprocal normal, for t in 2^-60 .. 2^126 and
// quotients that no format rounds to zero (2^-18 and up); below, CUDA's division.
struct Divisor {
    float t, r;
    bool slow;
    __device__ __forceinline__ explicit Divisor(float by) {
        t = by;
        r = __frcp_rn(by);
        slow = by < 8.67361738e-19f;        // 2^-60
    }
    __device__ __forceinline__ void apply(float (&v)[8]) const {
        if (slow) {
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = __fdiv_rn(v[i], t);
            return;
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            float q = __fmul_rn(v[i], r);
            q = __fmaf_rn(__fmaf_rn(-t, q, v[i]), r, q);
            v[i] = __fmaf_rn(__fmaf_rn(-t, q, v[i]), r, q);
        }
    }
};
__device__ __forceinline__ uint2 codes_e4m3(const float (&v)[8]) {
    unsigned short c[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(c[i]) : "f"(v[2 * i + 1]), "f"(v[2 * i]));
    return make_uint2(c[0] | uint32_t(c[1]) << 16, c[2] | uint32_t(c[3]) << 16);
}
__device__ __forceinline__ uint2 codes_e5m2(const float (&v)[8]) {
    unsigned short c[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) asm("cvt.rn.satfinite.e5m2x2.f32 %0, %1, %2;" : "=h"(c[i]) : "f"(v[2 * i + 1]), "f"(v[2 * i]));
    return make_uint2(c[0] | uint32_t(c[1]) << 16, c[2] | uint32_t(c[3]) << 16);
}
__device__ __forceinline__ uint32_t codes_e2m1(const float (&v)[8]) {           // element 2i in the low nibble of byte i
    uint32_t w;
    asm("{\n\t.reg .b8 a, b, c, d;\n\tcvt.rn.satfinite.e2m1x2.f32 a, %2, %1;\n\tcvt.rn.satfinite.e2m1x2.f32 b, %4, %3;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 c, %6, %5;\n\tcvt.rn.satfinite.e2m1x2.f32 d, %8, %7;\n\tmov.b32 %0, {a, b, c, d};\n\t}"
        : "=r"(w) : "f"(v[0]), "f"(v[1]), "f"(v[2]), "f"(v[3]), "f"(v[4]), "f"(v[5]), "f"(v[6]), "f"(v[7]));
    return w;
}
// E8M0 code of a block from the bits of its largest magnitude, and 2^(127 - code): a block of zeros gets 0, one with an infinity or NaN 255.
__device__ __forceinline__ uint32_t e8m0_code(uint32_t amax_bits, int emax) {
    const int e = int(amax_bits >> 23);
    return e == 255 ? 255u : uint32_t(max(e - emax, 0));
}
__device__ __forceinline__ float e8m0_inverse(uint32_t code) { return __uint_as_float(code == 255u ? 0x7FC00000u : (254u - code) << 23); }
// UE4M3 code nearest to x in 2^-9 .. 448 (NaN: 0x7F), and its value.
__device__ __forceinline__ uint32_t ue4m3_code(float x) {
    unsigned short c;
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(c) : "f"(0.0f), "f"(x));
    return max(uint32_t(c) & 0x7Fu, 1u);
}
__device__ __forceinline__ float ue4m3_value(uint32_t code) {
    uint32_t h;
    asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h) : "h"((unsigned short)code));
    return __half2float(__ushort_as_half((unsigned short)h));
}

}  // namespace quant
}  // namespace mmasim
