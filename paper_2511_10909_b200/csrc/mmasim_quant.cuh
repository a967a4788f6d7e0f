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

// Eight FP32 numbers as four pairs: additions, products and multiply-adds of pairs are one instruction each.
using Pair = unsigned long long;
__device__ __forceinline__ Pair pair(float a, float b) { Pair r; asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b)); return r; }
__device__ __forceinline__ Pair both(float a) { return pair(a, a); }
__device__ __forceinline__ void split(Pair p, float& a, float& b) { asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(p)); }
__device__ __forceinline__ Pair add2(Pair a, Pair b) { Pair r; asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b)); return r; }
__device__ __forceinline__ Pair mul2(Pair a, Pair b) { Pair r; asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b)); return r; }
__device__ __forceinline__ Pair fma2(Pair a, Pair b, Pair c) { Pair r; asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c)); return r; }
__device__ __forceinline__ Pair fma2_down(Pair a, Pair b, Pair c) { Pair r; asm("fma.rm.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c)); return r; }

template <int T> __device__ __forceinline__ void widen(const Raw<T>& r, Pair (&v)[4]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if constexpr (T == EF_F32) v[i] = pair(__uint_as_float(r.w[2 * i]), __uint_as_float(r.w[2 * i + 1]));
        else if constexpr (T == EF_BF16) v[i] = pair(__uint_as_float(r.w[i] << 16), __uint_as_float(r.w[i] & 0xFFFF0000u));
        else {
            const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&r.w[i]));
            v[i] = pair(f.x, f.y);
        }
    }
}
template <int T> __device__ __forceinline__ void narrow(const Pair (&v)[4], Raw<T>& r) {        // to nearest, once
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        float a, b;
        split(v[i], a, b);
        if constexpr (T == EF_F32) { r.w[2 * i] = __float_as_uint(a); r.w[2 * i + 1] = __float_as_uint(b); }
        else if constexpr (T == EF_BF16) asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r.w[i]) : "f"(b), "f"(a));
        else asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r.w[i]) : "f"(b), "f"(a));
    }
}
// a + b, rounded once to the rows' type.
template <int T> __device__ __forceinline__ void add_to(Raw<T>& a, const Raw<T>& b) {
#pragma unroll
    for (int i = 0; i < Elem<T>::WORDS; ++i) {
        if constexpr (T == EF_F32) a.w[i] = __float_as_uint(__fadd_rn(__uint_as_float(a.w[i]), __uint_as_float(b.w[i])));
        else if constexpr (T == EF_BF16) asm("add.rn.bf16x2 %0, %0, %1;" : "+r"(a.w[i]) : "r"(b.w[i]));
        else asm("add.rn.f16x2 %0, %0, %1;" : "+r"(a.w[i]) : "r"(b.w[i]));
    }
}
// The first `n` of eight elements, the rest zeros.  VEC: all eight or none, at a multiple of 16 bytes; else n may be anything, `vec` says
// whether the address is such a multiple.
template <int T, bool VEC> __device__ __forceinline__ Raw<T> load8(const typename Elem<T>::type* p, int n, bool vec) {
    Raw<T> r;
    if ((VEC || vec) && n >= 8) {
#pragma unroll
        for (int i = 0; i < Elem<T>::WORDS; i += 4) {
            const uint4 q = reinterpret_cast<const uint4*>(p)[i / 4];
            r.w[i] = q.x; r.w[i + 1] = q.y; r.w[i + 2] = q.z; r.w[i + 3] = q.w;
        }
    } else if constexpr (VEC) {
#pragma unroll
        for (int i = 0; i < Elem<T>::WORDS; ++i) r.w[i] = 0u;
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
template <int T, bool VEC> __device__ __forceinline__ void store8(typename Elem<T>::type* p, const Raw<T>& r, int n, bool vec) {      // n > 0
    if (VEC || (vec && n >= 8)) {
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
// Eight elements `step` apart (of `n` left in the row): for rows that no 16-byte access fits, where neighbouring threads take neighbouring
// elements.
template <int T> __device__ __forceinline__ Raw<T> load_spread(const typename Elem<T>::type* p, int n, int step) {
    Raw<T> r;
    if constexpr (T == EF_F32) {
#pragma unroll
        for (int i = 0; i < 8; ++i) r.w[i] = i * step < n ? __float_as_uint(p[i * step]) : 0u;
    } else {
        const unsigned short* s = reinterpret_cast<const unsigned short*>(p);
#pragma unroll
        for (int i = 0; i < 4; ++i) r.w[i] = (2 * i * step < n ? uint32_t(s[2 * i * step]) : 0u) | (2 * i * step + step < n ? uint32_t(s[2 * i * step + step]) << 16 : 0u);
    }
    return r;
}
template <int T> __device__ __forceinline__ void store_spread(typename Elem<T>::type* p, const Raw<T>& r, int n, int step) {
    if constexpr (T == EF_F32) {
#pragma unroll
        for (int i = 0; i < 8; ++i) if (i * step < n) p[i * step] = __uint_as_float(r.w[i]);
    } else {
        unsigned short* s = reinterpret_cast<unsigned short*>(p);
#pragma unroll
        for (int i = 0; i < 8; ++i) if (i * step < n) s[i * step] = (unsigned short)(i & 1 ? r.w[i / 2] >> 16 : r.w[i / 2]);
    }
}
template <int T> __device__ __forceinline__ void load_weight_spread(const void* w, bool f32, int at, int n, int step, Pair (&v)[4]) {
    if (!w) {
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = both(1.0f);
    } else if (f32) widen<EF_F32>(load_spread<EF_F32>(static_cast<const float*>(w) + at, n, step), v);
    else widen<T>(load_spread<T>(static_cast<const typename Elem<T>::type*>(w) + at, n, step), v);
}
// Eight weights of a norm: of the rows' type or FP32, or ones.
template <int T, bool VEC> __device__ __forceinline__ void load_weight8(const void* w, bool f32, int at, int n, bool vec, Pair (&v)[4]) {
    if (!w) {
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = both(1.0f);
    } else if (f32) widen<EF_F32>(load8<EF_F32, VEC>(static_cast<const float*>(w) + at, n, vec), v);
    else widen<T>(load8<T, VEC>(static_cast<const typename Elem<T>::type*>(w) + at, n, vec), v);
}
// 1 / sqrt(x) for x >= 0: the approximation and one step of Newton's method (within 2^-23); of infinity 0, of 0 and NaN not finite.
__device__ __forceinline__ float inverse_root(float x) {
    const float r = rsqrtf(x);
    const float e = __fmaf_rn(-__fmul_rn(x, r), r, 1.0f);
    return x < __uint_as_float(INF_BITS) ? __fmaf_rn(__fmul_rn(0.5f, r), e, r) : r;
}

// ---- codes ----
// The largest of `top` and the magnitudes of eight numbers, as bits: a NaN among them is the largest, then infinity.
__device__ __forceinline__ uint32_t largest(uint32_t top, const Pair (&v)[4]) {
    float m = __uint_as_float(top);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        float a, b;
        split(v[i], a, b);
        asm("max.NaN.abs.f32 %0, %0, %1, %2;" : "+f"(m) : "f"(a), "f"(b));
    }
    return __float_as_uint(m);
}
// The same of elements as loaded; `m` holds the largest of each half so far (16-bit types), largest_of puts them together.
template <int T> __device__ __forceinline__ void largest_halves(uint32_t& m, const Raw<T>& r) {
#pragma unroll
    for (int i = 0; i < Elem<T>::WORDS; ++i) {
        if constexpr (T == EF_F32) m = max(m, r.w[i] & 0x7FFFFFFFu);
        else if constexpr (T == EF_BF16) asm("max.NaN.bf16x2 %0, %0, %1;" : "+r"(m) : "r"(r.w[i] & 0x7FFF7FFFu));
        else asm("max.NaN.f16x2 %0, %0, %1;" : "+r"(m) : "r"(r.w[i] & 0x7FFF7FFFu));
    }
}
template <int T> __device__ __forceinline__ uint32_t largest_of(uint32_t m) {
    if constexpr (T == EF_F32) return m;
    else if constexpr (T == EF_BF16) return max(m << 16, m & 0xFFFF0000u);
    else {
        const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&m));
        return max(__float_as_uint(f.x), __float_as_uint(f.y));
    }
}
// x / t as the product with the reciprocal, corrected by its exact remainder (Markstein, Computation of elementary functions on the IBM RISC
// System/6000, 1990): a quotient that is an FP32 number comes out exactly, so that ties of the codes stay ties, every other one as division
// rounds it unless it lies within 2^-21 of a unit in the last place from the middle of two numbers.  No code changes with those: only where one of
// the two numbers is a tie of the codes could one, such divisors and dividends are few (a tie has at most four bits behind the leading one), and
// with a reciprocal known to a unit the only pair of them to come out otherwise has a divisor of 24 ones, for which it does not either
// (tests/test_gpu_quotients.py goes through them all).  For t in 2^-60 .. 2^126, where the
// remainder of a quotient that no format rounds to zero (2^-18 and up) is exact and the reciprocal normal; below, CUDA's division.
// A remainder of nothing is -0 (rounding down; it is exact otherwise), which leaves a quotient of zero its sign.
// (Its reciprocal and a second correction, exact for every quotient, made NVFP4 4096 x 4096 14.8 us where it took 13.4 without.)
struct Divisor {
    float t, r;
    bool slow;
    __device__ __forceinline__ explicit Divisor(float by) {
        t = by;
        asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(by));
        r = __fmaf_rn(__fmaf_rn(-by, r, 1.0f), r, r);
        slow = by < 8.67361738e-19f;        // 2^-60
    }
    __device__ __forceinline__ float operator()(float x) const {
        const float q = __fmul_rn(x, r);
        return slow ? __fdiv_rn(x, t) : __fmaf_rn(__fmaf_rd(-t, q, x), r, q);
    }
    __device__ __forceinline__ void apply(Pair (&v)[4]) const {
        if (slow) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                float a, b;
                split(v[i], a, b);
                v[i] = pair(__fdiv_rn(a, t), __fdiv_rn(b, t));
            }
            return;
        }
        const Pair rr = both(r), tt = both(-t);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const Pair q = mul2(v[i], rr);
            v[i] = fma2(fma2_down(tt, q, v[i]), rr, q);
        }
    }
};
__device__ __forceinline__ uint2 codes_e4m3(const Pair (&v)[4]) {
    unsigned short c[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        float a, b;
        split(v[i], a, b);
        asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(c[i]) : "f"(b), "f"(a));
    }
    return make_uint2(c[0] | uint32_t(c[1]) << 16, c[2] | uint32_t(c[3]) << 16);
}
__device__ __forceinline__ uint2 codes_e5m2(const Pair (&v)[4]) {
    unsigned short c[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        float a, b;
        split(v[i], a, b);
        asm("cvt.rn.satfinite.e5m2x2.f32 %0, %1, %2;" : "=h"(c[i]) : "f"(b), "f"(a));
    }
    return make_uint2(c[0] | uint32_t(c[1]) << 16, c[2] | uint32_t(c[3]) << 16);
}
__device__ __forceinline__ uint32_t codes_e2m1(const Pair (&p)[4]) {           // element 2i in the low nibble of byte i
    uint32_t w;
    float v[8];
#pragma unroll
    for (int i = 0; i < 4; ++i) split(p[i], v[2 * i], v[2 * i + 1]);
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
