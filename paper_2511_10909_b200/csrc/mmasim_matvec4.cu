// Products of a few tokens with 4-bit weights and group scales (mmasim_matvec4), weights as the group-scaled products take them (MXF4, NVF4):
//
//   y[t, n] = row_scale[n] * sum over k of x[t, k] * e2m1(W[n, k]) * sf[n, k / kb]          in FP32
//
// What should bound it is reading the weights once: 46 of them per clock and SM at the memory's rate.  The products go to the warp-level matrix
// instruction (exact products, FP32 sums), 16 rows of weights against columns of x, so that a weight costs its decoding and little else: one
// conversion into FP16 for two codes.  The scales multiply
//   - sums, where the tokens are few (one or two of 16 bits): a token has four of the instruction's eight columns, one for each of the four
//     blocks of 32 that a warp's lanes have of 128 elements, so that sums come by block (BlockProduct);
//   - weights, else: one multiplication for two, exact in FP16 (E2M1 times UE4M3 has six bits; the E8M0 scales of four neighbouring blocks enter
//     relative to their largest, which multiplies the sum) (Product).
// 256 elements of 16 rows take a warp 274 instructions the first way (NVFP4, one token) and 337 the second.
//
// x is staged once per CTA in shared memory, a column of FP16 numbers per token (FP32: three, each with what the one before left), scaled by a
// power of two per 128 elements so that the largest is in 2^14 .. 2^15.  Elements down to 2^-28 of the largest of their 128 are normal FP16 numbers
// that way (smaller ones, as subnormal numbers, the instruction would align as if they were 2^-14, and cut off bits of a sum of such alone), and
// then exact.  256 elements of which one is neither that nor zero go another way, from x itself: BF16 through the instruction's BF16 form and
// its wider exponents, with the codes moved to the lowest bits of a BF16 word's exponent - a number 2^-126 times its value; FP32 through plain
// multiply-adds (three parts in BF16 end at 2^-133, where FP32 elements below 2^-110 have bits that count).
// The instruction's sums truncate below 2^-24 of their largest term, so they are taken over 128 elements and added up in FP32.
//
// One CTA an SM walks over tiles of 16 rows; its warps split K (256 elements in turn) among the 16, 8, 4 or 2 of them that share a tile, by
// how many tiles are left, so that the last ones are spread over the whole chip.  Every warp has the loads of its next three steps in flight
// into its own part of shared memory, over the ends of tiles too (28672 x 8192: 49 us with these asynchronous copies where loads into registers,
// as far ahead, took 66).
// Where it ends: 28672 x 8192 NVFP4, one token, 29.5 us, 0.69 of the copy rate (the copies alone 25.7: 2.5 us until x is staged and the first
// tile begun, 7 % for tiles that do not fill the last round; then 2.6 instructions per clock and scheduler quarter).
#include <type_traits>
#include "mmasim_quant.cuh"

namespace mmasim {
namespace {
using namespace quant;

constexpr int ROWS = 16, STEP = 256, HALF = 128;        // elements of K that a warp takes at a time, and that share a scale of x
constexpr int WARPS = 16;                   // of a CTA, the only one of its SM
constexpr int STAGE = 2304;                 // bytes of a warp's loads of one step: two blocks of 32 weights of two rows for every lane, 16 rows' scale codes
constexpr int BLOCK_TOKENS = 2;             // up to so many tokens in columns by block
constexpr size_t SMEM_MOST = 227 * 1024;

template <int T> constexpr int PARTS = T == EF_F32 ? 3 : 1;

// Places in shared memory: x, a step of zeros, the scales of the columns, by token the steps that are not exact in FP16, the warps' shares of
// a tile, their loads in flight.  (What the host works out here it need not at the start of every CTA.)
struct Layout {
    int steps, pitch;                       // pitch: bytes of a column
    uint32_t zeros, scales, flags, share, ring;
};
// A column has HALF_BYTES per 128 elements: four blocks of 32, 16 bytes more behind two of them, and columns 32 bytes off a multiple of 128, so
// that the eight lanes of a quarter warp (four blocks of two columns) read from different banks.
constexpr int HALF_BYTES = HALF * 2 + 16;
__host__ __device__ constexpr int block_at(int half, int block) { return half * HALF_BYTES + block * 64 + (block >> 1) * 16; }
constexpr size_t layout(int K, int columns, int nt, int stages, Layout* l) {
    l->steps = (K + STEP - 1) / STEP;
    l->pitch = (l->steps * (STEP / HALF) * HALF_BYTES + 95) / 128 * 128 + 32;
    const size_t zeros = size_t(columns) * l->pitch, scales = zeros + 2 * HALF_BYTES, flags = scales + size_t(l->steps) * (STEP / HALF) * nt * 8 * 4;
    const size_t share = (flags + size_t(columns) * l->steps + 15) / 16 * 16, ring = share + size_t(WARPS) * ROWS * nt * 8 * 4;
    l->zeros = uint32_t(zeros); l->scales = uint32_t(scales); l->flags = uint32_t(flags); l->share = uint32_t(share); l->ring = uint32_t(ring);
    return ring + size_t(stages) * WARPS * STAGE;
}
constexpr size_t least_layout(int64_t K, int columns) {
    Layout l = {};
    return layout(int(K), columns, 1, 2, &l);
}
static_assert(least_layout(ROWS_MAX_K, PARTS<EF_BF16>) <= SMEM_MOST && least_layout(MATVEC_MAX_K_F32, PARTS<EF_F32>) <= SMEM_MOST, "one token of the longest rows fits");

struct MatvecArgs {
    int N, K, tokens;
    const uint8_t *w, *sf;
    const float* row_scale;
    const void* x;
    void* y;
    int64_t ldw, ldx, ldy;                  // ldw in bytes
    int vec_x, stages, copy_codes;
    int tiles, chunks;                      // of 16 rows, and of 32 elements of K
    Layout l;
};

// The tiles and steps of a warp, one after the other: rounds in which groups of `split` warps have a tile each.
struct Walk {
    int done, split, tile, part, base;      // this warp's step is base + part, base in steps of split
    __device__ __forceinline__ void begin(int d, int tiles, int ctas) {
        done = d;
        const int rest = tiles - done, warp = threadIdx.x >> 5;
        split = rest > 7 * ctas ? WARPS / 8 : (rest > 3 * ctas ? WARPS / 4 : (rest > ctas ? WARPS / 2 : WARPS));
        const int group = warp / split;
        tile = done + group * ctas + blockIdx.x;
        part = warp - group * split;
        base = 0;
    }
    __device__ __forceinline__ int step() const { return base + part; }
    __device__ __forceinline__ int following(int ctas) const { return done + WARPS / split * ctas; }
};

struct Item {                               // a lane's blocks of 32 weights of two rows, and their scale codes
    uint4 a, b;
    uint32_t ca, cb;
};
extern __shared__ __align__(128) unsigned char smem[];          // (places in it are 32-bit offsets)
__device__ __forceinline__ uint4 load16(uint32_t at) { return *reinterpret_cast<const uint4*>(smem + at); }
// The codes of a block, and of two neighbouring ones (MXF4: in the halves of the word).
template <bool NV> __device__ __forceinline__ uint32_t load_code(const uint8_t* at) { return NV ? *reinterpret_cast<const unsigned short*>(at) : *at; }
template <bool NV> __device__ __forceinline__ uint32_t load_codes(const uint8_t* at) {
    return NV ? *reinterpret_cast<const uint32_t*>(at) : __byte_perm(*reinterpret_cast<const unsigned short*>(at), 0, 0x4140);
}

__device__ __forceinline__ uint32_t mul_f16x2(uint32_t a, uint32_t b) { uint32_t r; asm("mul.rn.f16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b)); return r; }
__device__ __forceinline__ uint32_t mul_bf16x2(uint32_t a, uint32_t b) { uint32_t r; asm("mul.rn.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b)); return r; }
__device__ __forceinline__ void decode_f16(uint32_t w, uint32_t (&r)[4]) {      // r[j]: codes 2j (low half) and 2j + 1
    asm("{\n\t.reg .b8 a, b, c, d;\n\tmov.b32 {a, b, c, d}, %4;\n\tcvt.rn.f16x2.e2m1x2 %0, a;\n\tcvt.rn.f16x2.e2m1x2 %1, b;\n\t"
        "cvt.rn.f16x2.e2m1x2 %2, c;\n\tcvt.rn.f16x2.e2m1x2 %3, d;\n\t}" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(w));
}
__device__ __forceinline__ void decode_bf16(uint32_t w, uint32_t (&r)[4]) {     // r[j]: codes j (low half) and j + 4, 2^-126 times their values
    const uint32_t u = w >> 8;
    r[0] = ((w & 0x000F000Fu) * 0x1040u) & 0x81C081C0u;
    r[1] = ((w & 0x00F000F0u) * 0x0104u) & 0x81C081C0u;
    r[2] = ((u & 0x000F000Fu) * 0x1040u) & 0x81C081C0u;
    r[3] = ((u & 0x00F000F0u) * 0x0104u) & 0x81C081C0u;
}
__device__ __forceinline__ void mma_first(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%10, %10, %10, %10};"
        : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1), "f"(0.0f));
}
template <bool BF16>
__device__ __forceinline__ void mma(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    if constexpr (BF16)
        asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
            : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
    else
        asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
            : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t word_of(const uint4& v, int i) { return i == 0 ? v.x : i == 1 ? v.y : i == 2 ? v.z : v.w; }
__device__ __forceinline__ float power(int code) { return __uint_as_float(code == 0 ? 0x00400000u : code == 255 ? 0x7FC00000u : uint32_t(code) << 23); }      // of an E8M0 code

// The value of the lowest four bits of c: they are the lowest of an FP32 word's exponent, a number 2^-126 times it.
__device__ __forceinline__ float code_value(uint32_t c) { return __fmul_rn(__uint_as_float((c & 8u) << 28 | (c & 7u) << 22), 8.50705917e37f); }
// A step that FP16 has not exactly, x from memory: four sums of the lane, of eight columns.
// FP32: every lane multiplies its blocks of two rows with the tokens themselves, whose sums go to the columns of their first parts.  Little of it
// at once: its registers come on top of the kernel's (all eight codes of a word unrolled 6.9 us, not 6.5, for one token of 4096 x 4096 without such steps).
template <bool NV>
__device__ __noinline__ float4 wide_sums_f32(uint4 va, uint4 vb, uint32_t ca, uint32_t cb, const float* x, int64_t ldx, int tokens, int first, int k) {
    constexpr int P = PARTS<EF_F32>;
    if (k < 0) va = vb = make_uint4(0u, 0u, 0u, 0u);     // (a block behind the last is the last again: infinite weights times zeros would be NaN)
    float d[4] = {};
#pragma unroll 1
    for (int tok = (first + P - 1) / P; tok < tokens && tok * P < first + 8; ++tok) {
        float sa = 0.0f, sb = 0.0f;
#pragma unroll 1
        for (int four = 0; four < 8; ++four) {
            const int shift = four & 1 ? 16 : 0;
            uint32_t wa = word_of(va, four >> 1) >> shift, wb = word_of(vb, four >> 1) >> shift;
            const float fa = NV ? ue4m3_value(ca >> (four & 4 ? 8 : 0) & 0x7Fu) : power(ca), fb = NV ? ue4m3_value(cb >> (four & 4 ? 8 : 0) & 0x7Fu) : power(cb);
            const Raw<EF_F32> v = load8<EF_F32, false>(x + (k >= 0 ? tok * ldx + k + four * 4 : 0), k >= 0 ? 4 : 0, false);
#pragma unroll
            for (int i = 0; i < 4; ++i, wa >>= 4, wb >>= 4) {
                sa = __fmaf_rn(__uint_as_float(v.w[i]), __fmul_rn(code_value(wa), fa), sa);
                sb = __fmaf_rn(__uint_as_float(v.w[i]), __fmul_rn(code_value(wb), fb), sb);
            }
        }
#pragma unroll
        for (int o = 1; o < 4; o *= 2) {
            sa = __fadd_rn(sa, __shfl_xor_sync(0xFFFFFFFFu, sa, o));
            sb = __fadd_rn(sb, __shfl_xor_sync(0xFFFFFFFFu, sb, o));
        }
        const int c = tok * P - first - 2 * int(threadIdx.x & 3);
        if (c == 0) { d[0] = sa; d[2] = sb; }
        if (c == 1) { d[1] = sa; d[3] = sb; }
    }
    return make_float4(d[0], d[1], d[2], d[3]);
}
// BF16, through the instruction.
template <bool NV, int PER_TOKEN>
__device__ __noinline__ float4 wide_sums_bf16(uint4 va, uint4 vb, uint32_t ca, uint32_t cb, const __nv_bfloat16* x, int64_t ldx, int vec_x, int tokens, int first, int k) {
    if (k < 0) va = vb = make_uint4(0u, 0u, 0u, 0u);
    uint32_t fa[2], fb[2], more_a = 0x3F803F80u, more_b = 0x3F803F80u;
    if constexpr (NV) {                                 // 2^118 times the scales: 2^126 times 448 would be too large
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            asm("cvt.rn.bf16x2.f32 %0, %1, %1;" : "=r"(fa[i]) : "f"(__fmul_rn(ue4m3_value(ca >> (8 * i) & 0x7Fu), 3.32306998946229e35f)));
            asm("cvt.rn.bf16x2.f32 %0, %1, %1;" : "=r"(fb[i]) : "f"(__fmul_rn(ue4m3_value(cb >> (8 * i) & 0x7Fu), 3.32306998946229e35f)));
        }
    } else {                                            // 2^126 times the scales, in two factors where one does not hold it
        fa[0] = fa[1] = ca == 255u ? 0x7FC07FC0u : (min(ca, 128u) + 126u) * 0x00800080u;
        fb[0] = fb[1] = cb == 255u ? 0x7FC07FC0u : (min(cb, 128u) + 126u) * 0x00800080u;
        if (ca != 255u && ca > 128u) more_a = (ca - 1u) * 0x00800080u;
        if (cb != 255u && cb > 128u) more_b = (cb - 1u) * 0x00800080u;
    }
    const int c = first + (int(threadIdx.x & 31) >> 2), tok = c / PER_TOKEN;
    const bool there = k >= 0 && tok < tokens && c % PER_TOKEN == 0;     // (a token's other columns: zeros)
    float d[4] = {};
#pragma unroll 1
    for (int word = 0; word < 4; ++word) {
        uint32_t ra[4], rb[4];
        decode_bf16(word_of(va, word), ra);
        decode_bf16(word_of(vb, word), rb);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            ra[j] = mul_bf16x2(mul_bf16x2(ra[j], fa[word >> 1]), more_a);
            rb[j] = mul_bf16x2(mul_bf16x2(rb[j], fb[word >> 1]), more_b);
        }
        const Raw<EF_BF16> v = load8<EF_BF16, false>(x + (there ? tok * ldx + k + word * 8 : 0), there ? 8 : 0, vec_x);
        // (the codes' order: elements j and j + 4 side by side)
        mma<true>(d, ra[0], rb[0], ra[1], rb[1], __byte_perm(v.w[0], v.w[2], 0x5410), __byte_perm(v.w[0], v.w[2], 0x7632));
        mma<true>(d, ra[2], rb[2], ra[3], rb[3], __byte_perm(v.w[1], v.w[3], 0x5410), __byte_perm(v.w[1], v.w[3], 0x7632));
    }
    constexpr float back = NV ? 256.0f : 1.0f;
    const int column = 2 * int(threadIdx.x & 3);
    const bool even = column % PER_TOKEN == 0, odd = (column + 1) % PER_TOKEN == 0;        // (of a column of zeros: NaN, where a weight is infinite)
    return make_float4(even ? d[0] * back : 0.0f, odd ? d[1] * back : 0.0f, even ? d[2] * back : 0.0f, odd ? d[3] * back : 0.0f);
}
// A step whose blocks have scales far apart or far out (or NaN), one block of the four at a time, for eight columns.
__device__ __noinline__ float4 block_sums(uint4 va, uint4 vb, int ca, int cb, uint32_t x, float2 f) {
    double sum[4] = {};
#pragma unroll 1
    for (int one = 0; one < 4; ++one) {
        const bool mine = int(threadIdx.x & 3) == one;
        const int from = int(threadIdx.x & 28) + one;
        const double pa = power(__shfl_sync(0xFFFFFFFFu, ca, from)), pb = power(__shfl_sync(0xFFFFFFFFu, cb, from));
        float d[4] = {};
#pragma unroll
        for (int word = 0; word < 4; ++word) {
            uint32_t ra[4], rb[4];
            decode_f16(mine ? word_of(va, word) : 0u, ra);
            decode_f16(mine ? word_of(vb, word) : 0u, rb);
            const uint4 b = load16(x + word * 16);
            mma<false>(d, ra[0], rb[0], ra[1], rb[1], b.x, b.y);
            mma<false>(d, ra[2], rb[2], ra[3], rb[3], b.z, b.w);
        }
        sum[0] += double(d[0]) * f.x * pa;
        sum[1] += double(d[1]) * f.y * pa;
        sum[2] += double(d[2]) * f.x * pb;
        sum[3] += double(d[3]) * f.y * pb;
    }
    return make_float4(float(sum[0]), float(sum[1]), float(sum[2]), float(sum[3]));
}

template <bool NV, int NT>
struct Product {
    uint32_t x[NT], scales_at;              // where this lane's block of the step is, in the column that it feeds, and the scales of the columns whose sums it has
    uint32_t x_next, scales_next;           // how far the following step is
    float acc[NT][4];

    __device__ __forceinline__ void begin(const Layout& l, int columns, int lane, int step, int split) {
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)     // (columns behind the last have its sums; nobody reads them)
            x[nt] = min(nt * 8 + (lane >> 2), columns - 1) * l.pitch + block_at(step * 2, lane & 3);
        scales_at = uint32_t(l.scales) + (lane & 3) * 8 + step * (2 * NT * 32);
        x_next = split * (2 * HALF_BYTES);
        scales_next = split * (2 * NT * 32);
    }
    __device__ __forceinline__ void next() {
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) x[nt] += x_next;
        scales_at += scales_next;
    }
    __device__ __forceinline__ float2 scales(int half, int nt) const { return *reinterpret_cast<const float2*>(smem + scales_at + (half * NT + nt) * 32); }
    __device__ __forceinline__ void add(int nt, const float4& v) {
        acc[nt][0] += v.x; acc[nt][1] += v.y; acc[nt][2] += v.z; acc[nt][3] += v.w;
    }
    // d[h] = 16 rows times the columns over each 128 of the step, weights times fa and fb (two halves of a block of 32 each); the two are
    // independent of one another, and so are the two sums of each, so that the instructions do not wait for one another.
    __device__ __forceinline__ void sums(const Item (&it)[2], const uint32_t (&fa)[2][2], const uint32_t (&fb)[2][2], float (&d)[2][NT][4]) const {
        float e[2][NT][4];
#pragma unroll
        for (int word = 0; word < 4; ++word) {
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                uint32_t ra[4], rb[4];
                decode_f16(word_of(it[h].a, word), ra);
                decode_f16(word_of(it[h].b, word), rb);
#pragma unroll
                for (int j = 0; j < 4; ++j) { ra[j] = mul_f16x2(ra[j], fa[h][word / 2]); rb[j] = mul_f16x2(rb[j], fb[h][word / 2]); }
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) {
                    const uint4 b = load16(x[nt] + h * HALF_BYTES + word * 16);
                    if (word == 0) {
                        mma_first(d[h][nt], ra[0], rb[0], ra[1], rb[1], b.x, b.y);
                        mma_first(e[h][nt], ra[2], rb[2], ra[3], rb[3], b.z, b.w);
                    } else {
                        mma<false>(d[h][nt], ra[0], rb[0], ra[1], rb[1], b.x, b.y);
                        mma<false>(e[h][nt], ra[2], rb[2], ra[3], rb[3], b.z, b.w);
                    }
                }
            }
        }
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int i = 0; i < 4; ++i) d[h][nt][i] = __fadd_rn(d[h][nt][i], e[h][nt][i]);
    }
    __device__ __forceinline__ void step_nv(const Item (&it)[2]) {
        float d[2][NT][4];
        uint32_t fa[2][2], fb[2][2];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            uint32_t sa, sb;
            asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(sa) : "h"((unsigned short)(it[h].ca & 0x7F7Fu)));
            asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(sb) : "h"((unsigned short)(it[h].cb & 0x7F7Fu)));
            fa[h][0] = __byte_perm(sa, sa, 0x1010); fa[h][1] = __byte_perm(sa, sa, 0x3232);
            fb[h][0] = __byte_perm(sb, sb, 0x1010); fb[h][1] = __byte_perm(sb, sb, 0x3232);
        }
        sums(it, fa, fb, d);
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
                const float2 f = scales(h, nt);
                acc[nt][0] = __fmaf_rn(d[h][nt][0], f.x, acc[nt][0]);
                acc[nt][1] = __fmaf_rn(d[h][nt][1], f.y, acc[nt][1]);
                acc[nt][2] = __fmaf_rn(d[h][nt][2], f.x, acc[nt][2]);
                acc[nt][3] = __fmaf_rn(d[h][nt][3], f.y, acc[nt][3]);
            }
    }
    // The scales of a row's four blocks enter relative to their largest: from 2^-14 on FP16 has the weights exactly.  Others, those outside
    // 2^-63 .. 2^102 (whose sums might leave FP32 before x's scale is applied) and NaN go the long way.
    __device__ __forceinline__ void step_mx(const Item (&it)[2]) {
        uint32_t fa[2][2], fb[2][2], top[2];
        bool fine = true;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const uint32_t c = it[h].ca << 16 | it[h].cb;
            top[h] = __vmaxu2(c, __shfl_xor_sync(0xFFFFFFFFu, c, 1));
            top[h] = __vmaxu2(top[h], __shfl_xor_sync(0xFFFFFFFFu, top[h], 2));
            const uint32_t up = c + 0x000F000Fu - top[h];           // (at least 1 in both halves where the scales are fine)
            fine = fine && it[h].ca + 14 >= top[h] >> 16 && it[h].cb + 14 >= (top[h] & 0xFFFFu) && (top[h] >> 16) - 64 <= 165 && (top[h] & 0xFFFFu) - 64 <= 165;
            fa[h][0] = fa[h][1] = (up >> 16) * 0x04000400u;
            fb[h][0] = fb[h][1] = (up & 0xFFFFu) * 0x04000400u;
        }
        if (!__all_sync(0xFFFFFFFFu, fine)) {
#pragma unroll 1
            for (int h = 0; h < 2; ++h) {
                const uint4 va = h ? it[1].a : it[0].a, vb = h ? it[1].b : it[0].b;
                const int ca = h ? it[1].ca : it[0].ca, cb = h ? it[1].cb : it[0].cb;
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) add(nt, block_sums(va, vb, ca, cb, x[nt] + h * HALF_BYTES, scales(h, nt)));
            }
            return;
        }
        float d[2][NT][4];
        sums(it, fa, fb, d);
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const float pa = __uint_as_float((top[h] & 0xFF0000u) << 7), pb = __uint_as_float(top[h] << 23);
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
                const float2 f = scales(h, nt);
                acc[nt][0] = __fmaf_rn(__fmul_rn(d[h][nt][0], pa), f.x, acc[nt][0]);
                acc[nt][1] = __fmaf_rn(__fmul_rn(d[h][nt][1], pa), f.y, acc[nt][1]);
                acc[nt][2] = __fmaf_rn(__fmul_rn(d[h][nt][2], pb), f.x, acc[nt][2]);
                acc[nt][3] = __fmaf_rn(__fmul_rn(d[h][nt][3], pb), f.y, acc[nt][3]);
            }
        }
    }
};

// The same for few tokens of 16 bits: a token has four columns, one for each of the four blocks of 32 of the 128 elements, with x there and
// zeros elsewhere.  The sums then come by block, and the scales multiply sums instead of weights: 8 products of a lane for 64.
template <bool NV, int NT>
struct BlockProduct {
    uint32_t x[NT], x_next[NT], scales_at, scales_next;         // where this lane's block of the step is (or zeros), how far the following one is
    float acc[NT][4];

    __device__ __forceinline__ void begin(const Layout& l, int columns, int lane, int step, int split) {
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            const int tok = nt * 2 + (lane >> 4), block = lane & 3;
            const bool own = (lane >> 2 & 3) == block && tok < columns;
            x[nt] = own ? tok * l.pitch + block_at(step * 2, block) : uint32_t(l.zeros);
            x_next[nt] = own ? split * (2 * HALF_BYTES) : 0;
        }
        scales_at = uint32_t(l.scales) + (lane >> 1 & 1) * 4 + step * (2 * NT * 32);
        scales_next = split * (2 * NT * 32);
    }
    __device__ __forceinline__ void next() {
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) x[nt] += x_next[nt];
        scales_at += scales_next;
    }
    __device__ __forceinline__ float scale(int half, int nt) const { return *reinterpret_cast<const float*>(smem + scales_at + half * (NT * 32) + nt * 8); }
    __device__ __forceinline__ void add(int nt, const float4& v) {
        acc[nt][0] += v.x; acc[nt][1] += v.y; acc[nt][2] += v.z; acc[nt][3] += v.w;
    }
    // d[h][s]: of the two sixteens of the blocks of 32, weights without their scales
    __device__ __forceinline__ void sums(const uint4 (&wa)[2], const uint4 (&wb)[2], float (&d)[2][2][NT][4]) const {
#pragma unroll
        for (int word = 0; word < 4; ++word)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                uint32_t ra[4], rb[4];
                decode_f16(word_of(wa[h], word), ra);
                decode_f16(word_of(wb[h], word), rb);
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) {
                    const uint4 b = load16(x[nt] + h * HALF_BYTES + word * 16);
                    float (&to)[4] = d[h][word / 2][nt];
                    if (word % 2 == 0) mma_first(to, ra[0], rb[0], ra[1], rb[1], b.x, b.y);
                    else mma<false>(to, ra[0], rb[0], ra[1], rb[1], b.x, b.y);
                    mma<false>(to, ra[2], rb[2], ra[3], rb[3], b.z, b.w);
                }
            }
    }
    // `codes`: of rows g (0) and g + 8 (1) for this lane's two columns, which are neighbouring blocks: NVF4 four bytes, MXF4 two in 16-bit halves
    __device__ __forceinline__ void step(const uint4 (&wa)[2], const uint4 (&wb)[2], const uint32_t (&codes)[2][2]) {
        float d[2][2][NT][4];
        sums(wa, wb, d);
        float s[2][2][2][2];                // [half][row][block][sixteen]
        if constexpr (NV) {
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int r = 0; r < 2; ++r) {
                    uint32_t lo, hi;
                    const uint32_t c = codes[h][r] & 0x7F7F7F7Fu;
                    asm("{\n\t.reg .b16 a, b;\n\tmov.b32 {a, b}, %2;\n\tcvt.rn.f16x2.e4m3x2 %0, a;\n\tcvt.rn.f16x2.e4m3x2 %1, b;\n\t}" : "=r"(lo), "=r"(hi) : "r"(c));
                    const float2 f0 = __half22float2(*reinterpret_cast<const __half2*>(&lo)), f1 = __half22float2(*reinterpret_cast<const __half2*>(&hi));
                    s[h][r][0][0] = f0.x; s[h][r][0][1] = f0.y;
                    s[h][r][1][0] = f1.x; s[h][r][1][1] = f1.y;
                }
        } else {
            uint32_t least = codes[0][0], most = least;
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int r = 0; r < 2; ++r) {
                    least = __vminu2(least, codes[h][r]);
                    most = __vmaxu2(most, codes[h][r]);
                    s[h][r][0][0] = __uint_as_float(codes[h][r] << 23);
                    s[h][r][1][0] = __uint_as_float(codes[h][r] << 7 & 0x7F800000u);
                }
            // scales outside 2^-63 .. 2^102, whose products with the sums might leave FP32 before x's scale is applied, the smallest, and NaN
            if ((least & 0xFFFFu) < 64 || least >> 16 < 64 || (most & 0xFFFFu) > 229 || most >> 16 > 229) {
#pragma unroll
                for (int h = 0; h < 2; ++h)
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt) {
                        const double f = scale(h, nt);
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            const double v = (double(d[h][0][nt][i]) + double(d[h][1][nt][i])) * f * power(codes[h][i >> 1] >> (i & 1 ? 16 : 0) & 0xFFu);
                            acc[nt][i] += float(v);
                        }
                    }
                return;
            }
        }
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
                const float f = scale(h, nt);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float (&by)[2] = s[h][i >> 1][i & 1];
                    const float v = NV ? __fmaf_rn(d[h][0][nt][i], by[0], __fmul_rn(d[h][1][nt][i], by[1])) : __fmul_rn(__fadd_rn(d[h][0][nt][i], d[h][1][nt][i]), by[0]);
                    acc[nt][i] = __fmaf_rn(v, f, acc[nt][i]);
                }
            }
    }
};

__device__ __forceinline__ void copy16(uint32_t to, const void* from) { asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" :: "r"(to), "l"(from) : "memory"); }
__device__ __forceinline__ void copy8(uint32_t to, const void* from) { asm volatile("cp.async.ca.shared.global [%0], [%1], 8;" :: "r"(to), "l"(from) : "memory"); }
// Eight elements of a token into its columns, scaled with the others of their 128 (16 threads); false if one of them is not exact in FP16.
template <int T>
__device__ __forceinline__ bool stage_x(const Raw<T>& raw, unsigned char* at, int pitch, float* scale) {
    constexpr int P = PARTS<T>;
    if constexpr (T == EF_F16) {
        *reinterpret_cast<uint4*>(at) = make_uint4(raw.w[0], raw.w[1], raw.w[2], raw.w[3]);
        if (scale) *scale = 1.0f;
        return true;
    } else {
        Pair p[4];
        widen<T>(raw, p);
        uint32_t top = largest(0u, p);
#pragma unroll
        for (int s = 8; s > 0; s >>= 1) top = max(top, __shfl_xor_sync(0xFFFFFFFFu, top, s));
        // The largest times 2^up is in 2^14 .. 2^15, every part's scale a normal number, and no product with 2^up loses a bit (BF16; of FP32,
        // the parts behind would show it).
        const int up = min(141 - int(top >> 23), 126 - 12 * (P - 1));
        const Pair f = both(__uint_as_float(uint32_t(max(up, -126) + 127) << 23));
        uint32_t lost = up >= -16 && top < INF_BITS ? 0u : 1u, half[P][4], least = 0xFFFFFFFFu;           // least: of the magnitudes but zero, as bits, less one
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            float even, odd, x0, x1;
            split(p[j], x0, x1);
            split(mul2(p[j], f), even, odd);
            least = __viaddmin_u32(__float_as_uint(x0) & 0x7FFFFFFFu, 0xFFFFFFFFu, least);
            least = __viaddmin_u32(__float_as_uint(x1) & 0x7FFFFFFFu, 0xFFFFFFFFu, least);
#pragma unroll
            for (int q = 0; q < P; ++q) {
                asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(half[q][j]) : "f"(odd), "f"(even));
                if (P == 1) continue;                   // (a normal FP16 number has all bits of a BF16 one)
                const float2 back = __half22float2(*reinterpret_cast<const __half2*>(&half[q][j]));
                if (q == P - 1) lost |= (__float_as_uint(even) ^ __float_as_uint(back.x)) | (__float_as_uint(odd) ^ __float_as_uint(back.y));
                else {
                    even = __fmul_rn(__fsub_rn(even, back.x), 4096.0f);
                    odd = __fmul_rn(__fsub_rn(odd, back.y), 4096.0f);
                }
            }
        }
        lost |= uint32_t(least < (P > 1 || up < 113 ? uint32_t(113 - up) << 23 : 1u << (135 - up)) - 1u);          // times 2^up below 2^-14
#pragma unroll
        for (int q = 0; q < P; ++q) {
            *reinterpret_cast<uint4*>(at + q * pitch) = make_uint4(half[q][0], half[q][1], half[q][2], half[q][3]);
            if (scale) scale[q] = __uint_as_float(uint32_t(127 - max(up, -126) - 12 * q) << 23);
        }
        return lost == 0u;
    }
}

// What the parts of the kernel share.
template <int T, bool NV, int NT, bool BLOCKS>
struct Kernel {
    using E = typename Elem<T>::type;
    static constexpr int P = PARTS<T>, PER_TOKEN = BLOCKS ? 4 : P, CODES = NV ? 2 : 1, ROW_CODES = STEP / 32 * CODES, STEP_BYTES = STEP / 2;
    const MatvecArgs& a;
    const Layout& l;
    const int lane, warp, g, t, chunks, tiles, ctas;
    uint32_t ring, ring_end, in, out;                   // stages to be filled and to be read next
    Walk ahead;
    const uint8_t *wa, *wb, *codes;                     // of the step that is fetched next
    int w_next, codes_next;                             // bytes to the warp's following step

    __device__ __forceinline__ explicit Kernel(const MatvecArgs& args)
        : a(args), l(args.l), lane(threadIdx.x & 31), warp(threadIdx.x >> 5), g(lane >> 2), t(lane & 3), chunks(args.chunks), tiles(args.tiles), ctas(gridDim.x) {
        in = out = ring = l.ring + warp * (a.stages * STAGE);
        ring_end = ring + a.stages * STAGE;
        enter(0);
    }
    __device__ __forceinline__ void enter(int done) {   // (rows behind the last: it again, not stored)
        ahead.begin(done, tiles, ctas);
        const int first = (ahead.part * 8 + t) * 16;
        wa = a.w + min(ahead.tile * ROWS + g, a.N - 1) * a.ldw + first;
        wb = a.w + min(ahead.tile * ROWS + g + 8, a.N - 1) * a.ldw + first;
        codes = a.sf + int64_t(min(ahead.tile * ROWS + (lane & 15), a.N - 1)) * (chunks * CODES) + ahead.part * ROW_CODES;
        w_next = ahead.split * STEP_BYTES;
        codes_next = ahead.split * ROW_CODES;
    }
    // The next step's weights on their way: a lane copies what it will read itself, half a warp the codes.  GENERAL: of any K, the codes not
    // copied unless they can be.
    template <bool GENERAL> __device__ __forceinline__ void fetch() {
        if (ahead.done < tiles) {
            const int step = ahead.step();
            if (ahead.tile < tiles && step < l.steps) {
                const uint32_t to = uint32_t(__cvta_generic_to_shared(smem)) + in + lane * 16;
                int q = 0, r = 64;
                if (GENERAL && step == l.steps - 1) {   // (blocks behind the last: it again, times zeros of x)
                    q = (min(step * 8 + t, chunks - 1) - (step * 8 + t)) * 16;
                    r = (min(step * 8 + 4 + t, chunks - 1) - (step * 8 + t)) * 16;
                }
                copy16(to, wa + q);
                copy16(to + 512, wa + r);
                copy16(to + 1024, wb + q);
                copy16(to + 1536, wb + r);
                if (lane < 16 && (!GENERAL || a.copy_codes)) {
                    if constexpr (NV) copy16(to + 2048, codes);
                    else copy8(to + 2048 - lane * 8, codes);
                }
            }
            wa += w_next;
            wb += w_next;
            codes += codes_next;
            ahead.base += ahead.split;
            if (ahead.base >= l.steps) enter(ahead.following(ctas));
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
        in = in + STAGE == ring_end ? ring : in + STAGE;
    }
    // Its own copies of a warp's oldest step are there, the other lanes' too.
    __device__ __forceinline__ void await() const {
        if (a.stages == 4) asm volatile("cp.async.wait_group 3;" ::: "memory");
        else asm volatile("cp.async.wait_group 1;" ::: "memory");
        __syncwarp();
    }

    // x into its columns: a warp takes a step of a token at a time, 16 of its threads the 128 elements that share a scale.  The next two
    // are on their way meanwhile, asked for in front of the weights (28672 x 8192: 29.4 us, 30.0 with one; not at all where there are none, 4096 x
    // 4096 6.1 instead of 6.5).  Whether all of it is exact in FP16.
    static constexpr int BATCH = BLOCKS || T == EF_F32 ? 1 : 4;           // (more of few: more code to be fetched than there is to do)
    struct Steps {
        Raw<T> raw[BATCH];
        int tok, step;                                  // of the first, the others 16 steps apart
        __device__ __forceinline__ void settle(int steps) { while (step >= steps) { step -= steps; ++tok; } }
    };
    __device__ __forceinline__ void ask(Steps& s) const {
        s.settle(l.steps);
        int tok = s.tok, step = s.step;
#pragma unroll
        for (int i = 0; i < BATCH; ++i) {
            while (step >= l.steps) { step -= l.steps; ++tok; }
            const int k = step * STEP + lane * 8;
            const bool there = tok < a.tokens && k < a.K;
            s.raw[i] = load8<T, false>(static_cast<const E*>(a.x) + (there ? tok * a.ldx + k : 0), there ? 8 : 0, a.vec_x);
            step += WARPS;
        }
    }
    __device__ __forceinline__ void ask_behind(const Steps& s, Steps& following) const {
        following.tok = s.tok;
        following.step = s.step + BATCH * WARPS;
        ask(following);
    }
    __device__ __forceinline__ bool stage(Steps& s, Steps& next) {
        bool exact = true;
        while (s.tok < a.tokens) {
            Steps following;
            following.tok = a.tokens;
            if (next.tok < a.tokens) ask_behind(next, following);
#pragma unroll
            for (int i = 0; i < BATCH; ++i) {
                if (s.tok < a.tokens) {
                    const int half = s.step * 2 + (lane >> 4);
                    unsigned char* at = smem + s.tok * P * l.pitch + block_at(half, lane >> 2 & 3) + (lane & 3) * 16;
                    float* scale = (lane & 15) == 0 ? reinterpret_cast<float*>(smem + l.scales) + half * NT * 8 + s.tok * P : nullptr;
                    const bool lost = !__all_sync(0xFFFFFFFFu, stage_x<T>(s.raw[i], at, l.pitch, scale));
                    if (T != EF_F16 && lane == 0) smem[l.flags + s.tok * l.steps + s.step] = lost;
                    exact = exact && !lost;
                    s.step += WARPS;
                    s.settle(l.steps);
                }
            }
            s = next;
            next = following;
        }
        return exact;
    }
    // FP16 as it is, copied without a stop on the way.
    __device__ __forceinline__ void copy_x(Steps& s) const {
        for (s.settle(l.steps); s.tok < a.tokens; s.step += WARPS, s.settle(l.steps)) {
            const int half = s.step * 2 + (lane >> 4), k = s.step * STEP + lane * 8;
            unsigned char* at = smem + s.tok * P * l.pitch + block_at(half, lane >> 2 & 3) + (lane & 3) * 16;
            if (k < a.K) copy16(uint32_t(__cvta_generic_to_shared(at)), static_cast<const E*>(a.x) + s.tok * a.ldx + k);
            else *reinterpret_cast<uint4*>(at) = make_uint4(0, 0, 0, 0);
            if ((lane & 15) == 0) reinterpret_cast<float*>(smem + l.scales)[half * NT * 8 + s.tok * P] = 1.0f;
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
    }
    __device__ __forceinline__ bool inexact(int step) const {           // of any token
        bool lost = false;
        for (int tok = 0; tok < a.tokens; ++tok) lost = lost || smem[l.flags + tok * l.steps + step];
        return lost;
    }

    __device__ __forceinline__ float4 wide_sums(uint4 va, uint4 vb, uint32_t ca, uint32_t cb, int first, int k) const {
        const E* x = static_cast<const E*>(a.x);
        if constexpr (T == EF_F32) return wide_sums_f32<NV>(va, vb, ca, cb, x, a.ldx, a.tokens, first, k);
        else if constexpr (T == EF_BF16) return wide_sums_bf16<NV, PER_TOKEN>(va, vb, ca, cb, x, a.ldx, a.vec_x, a.tokens, first, k);
        else return make_float4(0.0f, 0.0f, 0.0f, 0.0f);            // (FP16 is always exact)
    }

    // The tile's shares of its warps, put together.
    __device__ __forceinline__ float row_scale(const Walk& now) const {        // of the row that this thread puts together (the same one for every token)
        const int first = threadIdx.x - warp / now.split * now.split * 32;
        return a.row_scale && first < ROWS * a.tokens && now.tile < tiles ? a.row_scale[min(now.tile * ROWS + (first & (ROWS - 1)), a.N - 1)] : 1.0f;
    }
    __device__ __forceinline__ void finish(const Walk& now, float scale, float (&acc)[NT][4]) const {
        constexpr int COLUMNS = BLOCKS ? NT * 2 : NT * 8;               // of a share
        float* const share = reinterpret_cast<float*>(smem + l.share);
        const int split = now.split, group = warp / split, bar = WARPS / split + group;         // barriers 1; 2, 3; 4 .. 7; 8 .. 15
        const int first = threadIdx.x - group * split * 32;
        float* mine = share + warp * (ROWS * COLUMNS);
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            if constexpr (BLOCKS) {                     // the four columns of a token are in two lanes
                float lo = __fadd_rn(acc[nt][0], acc[nt][1]), hi = __fadd_rn(acc[nt][2], acc[nt][3]);
                lo = __fadd_rn(lo, __shfl_xor_sync(0xFFFFFFFFu, lo, 1));
                hi = __fadd_rn(hi, __shfl_xor_sync(0xFFFFFFFFu, hi, 1));
                if (!(t & 1)) {
                    mine[g * COLUMNS + nt * 2 + (t >> 1)] = lo;
                    mine[(g + 8) * COLUMNS + nt * 2 + (t >> 1)] = hi;
                }
            } else {
                *reinterpret_cast<float2*>(mine + g * COLUMNS + nt * 8 + 2 * t) = make_float2(acc[nt][0], acc[nt][1]);
                *reinterpret_cast<float2*>(mine + (g + 8) * COLUMNS + nt * 8 + 2 * t) = make_float2(acc[nt][2], acc[nt][3]);
            }
            acc[nt][0] = acc[nt][1] = acc[nt][2] = acc[nt][3] = 0.0f;
        }
        asm volatile("bar.sync %0, %1;" :: "r"(bar), "r"(split * 32) : "memory");
        if (now.tile < tiles) {
            const float* shares = share + group * split * (ROWS * COLUMNS);
            for (int o = first; o < ROWS * a.tokens; o += split * 32) {
                const int r = o & (ROWS - 1), tok = o / ROWS, n = now.tile * ROWS + r;
                float v = 0.0f;
#pragma unroll
                for (int q = P - 1; q >= 0; --q) {      // the small parts first
                    const float* at = shares + r * COLUMNS + tok * P + q;
                    float s = 0.0f;
                    for (int w = 0; w < split; w += 2) s = __fadd_rn(s, __fadd_rn(at[w * (ROWS * COLUMNS)], at[(w + 1) * (ROWS * COLUMNS)]));
                    v = __fadd_rn(v, s);
                }
                if (n < a.N) {
                    v = __fmul_rn(v, scale);
                    E* y = static_cast<E*>(a.y) + tok * a.ldy + n;
                    if constexpr (T == EF_F32) *y = v;
                    else if constexpr (T == EF_BF16) *y = __float2bfloat16_rn(v);
                    else *y = __float2half_rn(v);
                }
            }
        }
        asm volatile("bar.sync %0, %1;" :: "r"(bar), "r"(split * 32) : "memory");
    }

    // GENERAL: of any K, codes from memory where they are not copied, steps that are not exact in FP16.
    template <bool GENERAL> __device__ __forceinline__ void run() {
        std::conditional_t<BLOCKS, BlockProduct<NV, NT>, Product<NV, NT>> product;
        Walk now;
        now.begin(0, tiles, ctas);
        float scale = row_scale(now);
        product.begin(l, a.tokens * P, lane, now.step(), now.split);
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) product.acc[nt][0] = product.acc[nt][1] = product.acc[nt][2] = product.acc[nt][3] = 0.0f;
        while (now.done < tiles) {
            __syncwarp();                               // (the codes of a stage are read by other lanes than copied them: all have read before it is filled again)
            fetch<GENERAL>();
            await();
            const int step = now.step();
            if (now.tile < tiles && step < l.steps) {
                const uint32_t at = out + lane * 16;
                const uint4 va[2] = {load16(at), load16(at + 512)}, vb[2] = {load16(at + 1024), load16(at + 1536)};
                // the codes of the blocks that the lane decodes (half, row), or that its sums are of
                const bool wide = GENERAL && T != EF_F16 && inexact(step), by_block = BLOCKS && !wide;
                uint32_t codes[2][2];
                const int block = by_block ? (t & 1) * 2 : t;
#pragma unroll
                for (int h = 0; h < 2; ++h)
#pragma unroll
                    for (int r = 0; r < 2; ++r) {
                        if (!GENERAL || a.copy_codes) {
                            const uint8_t* from = smem + out + 2048 + g * ROW_CODES + block * CODES + r * (8 * ROW_CODES) + h * (4 * CODES);
                            codes[h][r] = by_block ? load_codes<NV>(from) : load_code<NV>(from);
                        } else {
                            const uint8_t* from = a.sf + int64_t(min(now.tile * ROWS + g + r * 8, a.N - 1)) * (chunks * CODES);
                            const int q = step * 8 + 4 * h + block;
                            codes[h][r] = load_code<NV>(from + min(q, chunks - 1) * CODES);
                            if (by_block) codes[h][r] |= load_code<NV>(from + min(q + 1, chunks - 1) * CODES) << 16;
                        }
                    }
                if (wide) {
#pragma unroll 1
                    for (int h = 0; h < 2; ++h) {
                        const int k = step * STEP + h * HALF + t * 32;
#pragma unroll
                        for (int nt = 0; nt < NT; ++nt)
                            product.add(nt, wide_sums(h ? va[1] : va[0], h ? vb[1] : vb[0], h ? codes[1][0] : codes[0][0], h ? codes[1][1] : codes[0][1], nt * 8, k < a.K ? k : -1));
                    }
                } else if constexpr (BLOCKS) product.step(va, vb, codes);
                else {
                    const Item it[2] = {{va[0], vb[0], codes[0][0], codes[0][1]}, {va[1], vb[1], codes[1][0], codes[1][1]}};
                    if constexpr (NV) product.step_nv(it);
                    else product.step_mx(it);
                }
            }
            out = out + STAGE == ring_end ? ring : out + STAGE;
            now.base += now.split;
            product.next();
            if (now.base < l.steps) continue;
            finish(now, scale, product.acc);
            now.begin(now.following(ctas), tiles, ctas);
            scale = row_scale(now);
            product.begin(l, a.tokens * P, lane, now.step(), now.split);
        }
    }
};

// BLOCKS: of BlockProduct, a token has four columns of the instruction but one in shared memory.
template <int T, bool NV, int NT, bool BLOCKS>
__global__ void __launch_bounds__(WARPS * 32, 1) matvec4_kernel(const MatvecArgs a) {
    after_previous();
    Kernel<T, NV, NT, BLOCKS> k(a);
    // x is asked for before the weights' stream begins, and staged before more than a step a warp of it is in front.
    typename Kernel<T, NV, NT, BLOCKS>::Steps steps, next;
    steps.tok = 0;
    steps.step = k.warp;
    const bool as_it_is = T == EF_F16 && a.vec_x;
    if (as_it_is) k.copy_x(steps);
    else {
        k.ask(steps);
        next.tok = a.tokens;
        if (a.tokens * a.l.steps > k.BATCH * WARPS) k.ask_behind(steps, next);
    }
    const bool plain = a.K % STEP == 0 && a.copy_codes;
    if (plain) k.template fetch<false>();
    else k.template fetch<true>();
    if (BLOCKS && threadIdx.x < 2 * HALF_BYTES / 4) reinterpret_cast<uint32_t*>(smem + a.l.zeros)[threadIdx.x] = 0u;
    bool exact = true;
    if (as_it_is) asm volatile("cp.async.wait_group 1;" ::: "memory");
    else exact = k.stage(steps, next);
    const bool wide = __syncthreads_or(!exact);
    for (int i = 2; i < a.stages; ++i) {
        if (plain) k.template fetch<false>();
        else k.template fetch<true>();
    }
    if (plain && !wide) k.template run<false>();
    else k.template run<true>();
}

template <int T, bool NV, int NT, bool BLOCKS>
cudaError_t launch(const MatvecArgs& a, size_t smem, cudaStream_t stream) {
    if (smem > 48 * 1024) {
        const cudaError_t err = cudaFuncSetAttribute(matvec4_kernel<T, NV, NT, BLOCKS>, cudaFuncAttributeMaxDynamicSharedMemorySize, int(SMEM_MOST));
        if (err != cudaSuccess) { cudaGetLastError(); return err; }
    }
    return enqueue(matvec4_kernel<T, NV, NT, BLOCKS>, dim3(unsigned(a.tiles < 148 ? a.tiles : 148)), WARPS * 32, smem, stream, a);
}
template <int T, bool NV>
cudaError_t launch(MatvecArgs a, int64_t all, int64_t bytes, cudaStream_t stream) {
    // tokens that read the weights together: 16 columns, as many as shared memory holds beside the shortest ring
    int most = 16 / PARTS<T>;
    while (layout(a.K, most * PARTS<T>, most * PARTS<T> > 8 ? 2 : 1, 2, &a.l) > SMEM_MOST) --most;
    const char *x = static_cast<const char*>(a.x), *y = static_cast<const char*>(a.y);
    cudaError_t err = cudaSuccess;
    most = int((all + (all + most - 1) / most - 1) / ((all + most - 1) / most));       // evenly
    for (int64_t done = 0; done < all && err == cudaSuccess; done += a.tokens) {
        a.tokens = int(all - done < most ? all - done : most);
        a.x = x + done * a.ldx * bytes;
        a.y = const_cast<char*>(y) + done * a.ldy * bytes;
        const int columns = a.tokens * PARTS<T>;
        const bool blocks = PARTS<T> == 1 && a.tokens <= BLOCK_TOKENS;
        const int nt = blocks || columns <= 8 ? 1 : 2;
        a.stages = layout(a.K, columns, nt, 4, &a.l) <= SMEM_MOST ? 4 : 2;
        const size_t smem = layout(a.K, columns, nt, a.stages, &a.l);
        if constexpr (PARTS<T> == 1) {
            static_assert(BLOCK_TOKENS * 4 <= 8, "a token by block has four of the instruction's eight columns");
            if (blocks) { err = launch<T, NV, 1, true>(a, smem, stream); continue; }
        }
        err = nt == 1 ? launch<T, NV, 1, false>(a, smem, stream) : launch<T, NV, 2, false>(a, smem, stream);
    }
    return err;
}
template <int T>
cudaError_t launch(bool nv, const MatvecArgs& a, int64_t tokens, int64_t bytes, cudaStream_t stream) {
    return nv ? launch<T, true>(a, tokens, bytes, stream) : launch<T, false>(a, tokens, bytes, stream);
}
}  // namespace

int launch_matvec4(bool nv, int fmt, int64_t T, int64_t N, int64_t K, const void* W, int64_t ldw, const void* sf, const float* row_scale,
                   const void* x, int64_t ldx, void* y, int64_t ldy, cudaStream_t stream) {
    const int64_t bytes = fmt == EF_F32 ? 4 : 2;
    MatvecArgs a = {};
    a.N = int(N); a.K = int(K);
    a.w = static_cast<const uint8_t*>(W);
    a.sf = static_cast<const uint8_t*>(sf);
    a.row_scale = row_scale;
    a.x = x; a.y = y;
    a.ldw = ldw / 2; a.ldx = ldx; a.ldy = ldy;
    a.tiles = (a.N + ROWS - 1) / ROWS;
    a.chunks = a.K / 32;
    a.copy_codes = K % STEP == 0 && reinterpret_cast<uintptr_t>(sf) % (nv ? 16 : 8) == 0;
    a.vec_x = (reinterpret_cast<uintptr_t>(x) | uintptr_t(ldx * bytes)) % 16 == 0;
    const cudaError_t err = fmt == EF_F32 ? launch<EF_F32>(nv, a, T, bytes, stream) : fmt == EF_BF16 ? launch<EF_BF16>(nv, a, T, bytes, stream) : launch<EF_F16>(nv, a, T, bytes, stream);
    if (err != cudaSuccess) { set_error("mmasim_matvec4: %s", cudaGetErrorString(err)); return MMASIM_ERR_CUDA; }
    return MMASIM_OK;
}

}  // namespace mmasim
