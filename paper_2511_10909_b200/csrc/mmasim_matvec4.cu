// Products of a few tokens with 4-bit weights and group scales (mmasim_matvec4), weights as the group-scaled products take them (MXF4, NVF4):
//
//   y[t, n] = row_scale[n] * sum over k of x[t, k] * e2m1(W[n, k]) * sf[n, k / kb]          in FP32
//
// What bounds it is reading the weights once: 46 of them per clock and SM at the memory's rate, when 64 lanes of integer work are to be had.
// So the products go to the warp-level matrix instruction (BF16, exact products, FP32 sums), and the work per weight is its decoding: a code
// s e e m moves to the sign and the lowest bits of a BF16 word's exponent and significand - a number 2^-126 times its value, subnormals and
// all - by one mask, one multiplication by two powers of two and one mask for two codes 16 bits apart; a multiplication by the scale times
// 2^126 (2^118 for UE4M3, whose range would not fit) makes it the weight, exactly: two bits times four at most.
// x is split into BF16 parts without a rounding (BF16 one, FP16 two, FP32 three), each a column of the instruction.  The instruction's sums
// truncate below 2^-25 of their largest term, so they are taken over 128 elements and added up in FP32 by rounding additions.
#include "mmasim_quant.cuh"

namespace mmasim {
namespace {
using namespace quant;

constexpr int WARPS = 8, ROWS = 16, SMEM_X = 32768;

struct MatvecArgs {
    int N, K, tokens;
    const uint8_t *w, *sf;
    const float* row_scale;
    const void* x;
    void* y;
    int64_t ldw, ldx, ldy;                  // ldw in bytes
    int slice;                              // chunks of 32 elements whose x is in shared memory at a time, a multiple of 4
    int vec_x;
};

// x = the sum of its BF16 parts: truncations of what is left (an infinity or NaN: the first part alone).
template <int PARTS> __device__ __forceinline__ void split(float v, uint32_t (&part)[PARTS]) {
#pragma unroll
    for (int p = 0; p < PARTS; ++p) {
        const uint32_t u = __float_as_uint(v);
        if ((u & 0x7F800000u) == 0x7F800000u) {
            part[p] = u >> 16 | (u & 0xFFFFu ? 0x40u : 0u);         // (a NaN stays one)
            v = 0.0f;
        } else {
            part[p] = u >> 16;
            v = __fsub_rn(v, __uint_as_float(u & 0xFFFF0000u));
        }
    }
}
__device__ __forceinline__ void decode(uint32_t w, uint32_t (&r)[4]) {          // r[j]: codes j (low half) and j + 4
    const uint32_t u = w >> 8;
    r[0] = ((w & 0x000F000Fu) * 0x1040u) & 0x81C081C0u;
    r[1] = ((w & 0x00F000F0u) * 0x0104u) & 0x81C081C0u;
    r[2] = ((u & 0x000F000Fu) * 0x1040u) & 0x81C081C0u;
    r[3] = ((u & 0x00F000F0u) * 0x0104u) & 0x81C081C0u;
}
__device__ __forceinline__ uint32_t mul2(uint32_t a, uint32_t b) {
    uint32_t r;
    asm("mul.rn.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
}
// E8M0 code -> 2^126 times its value as two equal BF16 words, in two factors where one does not hold it.
__device__ __forceinline__ void mx_scale(uint32_t code, uint32_t& a, uint32_t& b) {
    a = code == 255u ? 0x7FC07FC0u : (min(code, 128u) + 126u) * 0x00800080u;
    b = code == 255u || code <= 128u ? 0x3F803F80u : (code - 1u) * 0x00800080u;      // 2^(code - 128)
}
__device__ __forceinline__ uint32_t nv_scale(uint32_t code) {                       // UE4M3 code -> 2^118 times its value
    const float f = __fmul_rn(ue4m3_value(code & 0x7Fu), 3.32306998946229e35f);     // 2^118
    uint32_t r;
    asm("cvt.rn.bf16x2.f32 %0, %1, %1;" : "=r"(r) : "f"(f));
    return r;
}
__device__ __forceinline__ void mma(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

template <int T, bool NV>
__global__ void __launch_bounds__(WARPS * 32) matvec4_kernel(const MatvecArgs a) {
    using E = typename Elem<T>::type;
    constexpr int PARTS = T == EF_BF16 ? 1 : (T == EF_F16 ? 2 : 3);
    extern __shared__ __align__(128) unsigned char xs[];
    __shared__ float share[WARPS][ROWS][8];
    after_previous();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, g = lane >> 2, t = lane & 3;
    const int row0 = blockIdx.x * ROWS + g, ra = min(row0, a.N - 1), rb = min(row0 + 8, a.N - 1);       // (rows behind the last: read again, not stored)
    const int chunks = a.K / 32, columns = a.tokens * PARTS, pitch = a.slice * 64;
    const uint8_t *wa = a.w + ra * a.ldw, *wb = a.w + rb * a.ldw;
    const int per_row = NV ? chunks * 2 : chunks;
    const uint8_t *sa = a.sf + int64_t(ra) * per_row, *sb = a.sf + int64_t(rb) * per_row;
    float acc[4] = {0.0f, 0.0f, 0.0f, 0.0f};
    for (int c0 = 0; c0 < chunks; c0 += a.slice) {
        const int here = min(a.slice, chunks - c0), padded = (here + 3) / 4 * 4;
        if (c0) __syncthreads();
        for (int i = threadIdx.x; i < a.tokens * padded * 4; i += WARPS * 32) {         // x in the order of the codes' pairs
            const int tok = i / (padded * 4), q = i % (padded * 4) / 4, word = i & 3;
            float v[8];
            widen<T>(load8<T>(static_cast<const E*>(a.x) + tok * a.ldx + (q < here ? (c0 + q) * 32 + word * 8 : 0), q < here ? 8 : 0, a.vec_x), v);
            uint32_t part[8][PARTS];
#pragma unroll
            for (int e = 0; e < 8; ++e) split<PARTS>(v[e], part[e]);
#pragma unroll
            for (int p = 0; p < PARTS; ++p) {
                const int c = tok * PARTS + p;
                *reinterpret_cast<uint4*>(xs + c * pitch + q * 64 + ((word + q + c) & 3) * 16) =
                    make_uint4(part[0][p] | part[4][p] << 16, part[1][p] | part[5][p] << 16, part[2][p] | part[6][p] << 16, part[3][p] | part[7][p] << 16);
            }
        }
        __syncthreads();
        for (int s = warp; s * 4 < here; s += WARPS) {
            const int q = s * 4 + t;                    // this lane's chunk, of rows g and g + 8
            uint4 va = make_uint4(0, 0, 0, 0), vb = va;
            uint32_t ca = 0, cb = 0;
            if (q < here) {
                va = *reinterpret_cast<const uint4*>(wa + int64_t(c0 + q) * 16);
                vb = *reinterpret_cast<const uint4*>(wb + int64_t(c0 + q) * 16);
                if constexpr (NV) {
                    ca = reinterpret_cast<const unsigned short*>(sa)[c0 + q];
                    cb = reinterpret_cast<const unsigned short*>(sb)[c0 + q];
                } else {
                    ca = sa[c0 + q];
                    cb = sb[c0 + q];
                }
            }
            uint32_t fa[2], fb[2], more_a = 0x3F803F80u, more_b = 0x3F803F80u;
            if constexpr (NV) {
                fa[0] = nv_scale(ca); fa[1] = nv_scale(ca >> 8);
                fb[0] = nv_scale(cb); fb[1] = nv_scale(cb >> 8);
            } else {
                mx_scale(ca, fa[0], more_a);
                mx_scale(cb, fb[0], more_b);
                fa[1] = fa[0]; fb[1] = fb[0];
            }
            float d[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
            for (int word = 0; word < 4; ++word) {
                uint4 b = make_uint4(0, 0, 0, 0);
                if (g < columns) b = *reinterpret_cast<const uint4*>(xs + g * pitch + q * 64 + ((word + q + g) & 3) * 16);
                uint32_t wr[4], ws[4];
                decode(word == 0 ? va.x : word == 1 ? va.y : word == 2 ? va.z : va.w, wr);
                decode(word == 0 ? vb.x : word == 1 ? vb.y : word == 2 ? vb.z : vb.w, ws);
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    wr[j] = mul2(wr[j], fa[word / 2]);
                    ws[j] = mul2(ws[j], fb[word / 2]);
                    if constexpr (!NV) { wr[j] = mul2(wr[j], more_a); ws[j] = mul2(ws[j], more_b); }
                }
                mma(d, wr[0], ws[0], wr[1], ws[1], b.x, b.y);
                mma(d, wr[2], ws[2], wr[3], ws[3], b.z, b.w);
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) acc[i] = __fadd_rn(acc[i], d[i]);
        }
    }
    share[warp][g][2 * t] = acc[0];
    share[warp][g][2 * t + 1] = acc[1];
    share[warp][g + 8][2 * t] = acc[2];
    share[warp][g + 8][2 * t + 1] = acc[3];
    __syncthreads();
    for (int i = threadIdx.x; i < ROWS * a.tokens; i += WARPS * 32) {
        const int r = i % ROWS, tok = i / ROWS, n = blockIdx.x * ROWS + r;
        if (n >= a.N) continue;
        float v = 0.0f;
#pragma unroll
        for (int p = PARTS - 1; p >= 0; --p) {          // the small parts first
            float s = 0.0f;
#pragma unroll
            for (int w = 0; w < WARPS; ++w) s = __fadd_rn(s, share[w][r][tok * PARTS + p]);
            v = __fadd_rn(v, s);
        }
        if constexpr (NV) v = __fmul_rn(v, 256.0f);
        if (a.row_scale) v = __fmul_rn(v, a.row_scale[n]);
        E* y = static_cast<E*>(a.y) + tok * a.ldy + n;
        if constexpr (T == EF_F32) *y = v;
        else if constexpr (T == EF_BF16) *y = __float2bfloat16_rn(v);
        else *y = __float2half_rn(v);
    }
}

template <int T, bool NV>
cudaError_t launch(MatvecArgs a, int64_t T_all, int64_t bytes, cudaStream_t stream) {
    constexpr int PARTS = T == EF_BF16 ? 1 : (T == EF_F16 ? 2 : 3), MOST = 8 / PARTS;
    const char *x = static_cast<const char*>(a.x), *y = static_cast<const char*>(a.y);
    cudaError_t err = cudaSuccess;
    for (int64_t done = 0; done < T_all && err == cudaSuccess; done += MOST) {
        a.tokens = int(T_all - done < MOST ? T_all - done : MOST);
        a.x = x + done * a.ldx * bytes;
        a.y = const_cast<char*>(y) + done * a.ldy * bytes;
        const int columns = a.tokens * PARTS;
        a.slice = SMEM_X / (64 * columns) / 4 * 4;
        if (a.slice > (a.K / 32 + 3) / 4 * 4) a.slice = (a.K / 32 + 3) / 4 * 4;
        err = enqueue(matvec4_kernel<T, NV>, dim3(unsigned((a.N + ROWS - 1) / ROWS)), WARPS * 32, size_t(columns) * a.slice * 64, stream, a);
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
    a.vec_x = (reinterpret_cast<uintptr_t>(x) | uintptr_t(ldx * bytes)) % 16 == 0;
    const cudaError_t err = fmt == EF_F32 ? launch<EF_F32>(nv, a, T, bytes, stream) : fmt == EF_BF16 ? launch<EF_BF16>(nv, a, T, bytes, stream) : launch<EF_F16>(nv, a, T, bytes, stream);
    if (err != cudaSuccess) { set_error("mmasim_matvec4: %s", cudaGetErrorString(err)); return MMASIM_ERR_CUDA; }
    return MMASIM_OK;
}

}  // namespace mmasim
