// Gradients of the root-mean-square norm (mmasim_rms_norm_backward).  With r = 1 / sqrt(mean h^2 + eps) and g = dy w, by row:
//
//   dx = r g - h (r^3 / K) sum(g h) + dresidual         dweight = sum over rows of dy h r
//
// One pass: both sums of a row (h^2 and g h) come from the same loads, so nothing of the forward pass has to be kept but h.  Memory is what
// bounds it (8 bytes an element in BF16 with a residual).  A CTA walks over rows, a thread keeps its columns and with them its share of
// dweight in registers; the CTAs' shares go to the workspace, and a second kernel adds them column by column, in one order whatever runs first.
#include "mmasim_quant.cuh"

namespace mmasim {
namespace rows {
namespace {
using namespace quant;

constexpr int MAX_THREADS = 512;

struct BackArgs {
    int64_t M;
    int K, threads;
    const void *dy, *h, *w, *dres;
    void* dx;
    float* part;                            // gridDim.x rows of K, or NULL
    int64_t ld_dy, ld_h, ld_res, ld_dx;
    float eps, inverse_k;
    int w_f32, vec_dy, vec_h, vec_res, vec_dx, vec_w;
};

__device__ __forceinline__ float2 row_sums(float2 v, int threads, float2* slot) {
    for (int o = min(threads, 32) / 2; o > 0; o >>= 1) {
        v.x += __shfl_xor_sync(0xFFFFFFFFu, v.x, o);
        v.y += __shfl_xor_sync(0xFFFFFFFFu, v.y, o);
    }
    if (threads > 32) {
        if ((threadIdx.x & 31) == 0) slot[threadIdx.x >> 5] = v;
        __syncthreads();
        v = int(threadIdx.x & 15) < threads / 32 ? slot[threadIdx.x & 15] : make_float2(0.0f, 0.0f);
#pragma unroll
        for (int o = 8; o > 0; o >>= 1) {
            v.x += __shfl_xor_sync(0xFFFFFFFFu, v.x, o);
            v.y += __shfl_xor_sync(0xFFFFFFFFu, v.y, o);
        }
    }
    return v;
}

// HOLD: dy and h stay in registers between the sums and the results; else they are read again (rows too long for that).
template <int T, int V, bool HOLD, bool VEC>
__global__ void __launch_bounds__(MAX_THREADS) backward_kernel(const BackArgs a) {
    using E = typename Elem<T>::type;
    __shared__ float2 slots[2][16];
    __shared__ float group_share[8 * 128];
    after_previous();
    const int per_cta = a.threads > 32 ? 1 : int(blockDim.x) / a.threads;
    const int group = a.threads > 32 ? 0 : threadIdx.x / a.threads, t = a.threads > 32 ? threadIdx.x : threadIdx.x & (a.threads - 1);
    Pair dw[V][4];
#pragma unroll
    for (int j = 0; j < V; ++j)
#pragma unroll
        for (int i = 0; i < 4; ++i) dw[j][i] = 0;
    int turn = 0;
    for (int64_t first = int64_t(blockIdx.x) * per_cta; first < a.M; first += int64_t(gridDim.x) * per_cta, turn ^= 1) {
        const int64_t row = first + group;
        const int K = row < a.M ? a.K : 0;
        const E *dy = static_cast<const E*>(a.dy) + row * a.ld_dy, *h = static_cast<const E*>(a.h) + row * a.ld_h;
        Raw<T> dy_raw[HOLD ? V : 1], h_raw[HOLD ? V : 1], res_raw[HOLD ? V : 1];
        if constexpr (HOLD) {
#pragma unroll
            for (int j = 0; j < V; ++j) {
                const int at = (t + j * a.threads) * 8;
                h_raw[j] = load8<T, VEC>(h + at, K - at, a.vec_h);
                dy_raw[j] = load8<T, VEC>(dy + at, K - at, a.vec_dy);
                if (a.dres) res_raw[j] = load8<T, VEC>(static_cast<const E*>(a.dres) + row * a.ld_res + at, K - at, a.vec_res);
            }
        }
        Pair squares = 0, products = 0;
#pragma unroll
        for (int j = 0; j < V; ++j) {
            const int at = (t + j * a.threads) * 8;
            if constexpr (!HOLD) {
                h_raw[0] = load8<T, VEC>(h + at, K - at, a.vec_h);
                dy_raw[0] = load8<T, VEC>(dy + at, K - at, a.vec_dy);
            }
            Pair hv[4], g[4], w[4];
            widen<T>(h_raw[HOLD ? j : 0], hv);
            widen<T>(dy_raw[HOLD ? j : 0], g);
            load_weight8<T, VEC>(a.w, a.w_f32, at, K - at, a.vec_w, w);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                squares = fma2(hv[i], hv[i], squares);
                products = fma2(mul2(g[i], w[i]), hv[i], products);
            }
        }
        float2 sums, odd;
        split(squares, sums.x, odd.x);
        split(products, sums.y, odd.y);
        sums = row_sums(make_float2(sums.x + odd.x, sums.y + odd.y), a.threads, slots[turn]);          // (two sets of slots: one barrier a row)
        const float r = inverse_root(__fmaf_rn(sums.x, a.inverse_k, a.eps));
        const Pair rr = both(r), c = both(-__fmul_rn(__fmul_rn(__fmul_rn(__fmul_rn(r, r), r), sums.y), a.inverse_k));
#pragma unroll
        for (int j = 0; j < V; ++j) {
            const int at = (t + j * a.threads) * 8;
            if (at >= K) continue;
            if constexpr (!HOLD) {
                h_raw[0] = load8<T, VEC>(h + at, K - at, a.vec_h);
                dy_raw[0] = load8<T, VEC>(dy + at, K - at, a.vec_dy);
                if (a.dres) res_raw[0] = load8<T, VEC>(static_cast<const E*>(a.dres) + row * a.ld_res + at, K - at, a.vec_res);
            }
            Pair hv[4], g[4], w[4], out[4];
            widen<T>(h_raw[HOLD ? j : 0], hv);
            widen<T>(dy_raw[HOLD ? j : 0], g);
            load_weight8<T, VEC>(a.w, a.w_f32, at, K - at, a.vec_w, w);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                dw[j][i] = fma2(g[i], mul2(hv[i], rr), dw[j][i]);
                out[i] = fma2(mul2(g[i], w[i]), rr, mul2(hv[i], c));
            }
            if (a.dres) {
                Pair res[4];
                widen<T>(res_raw[HOLD ? j : 0], res);
#pragma unroll
                for (int i = 0; i < 4; ++i) out[i] = add2(out[i], res[i]);
            }
            Raw<T> o;
            narrow<T>(out, o);
            store8<T, VEC>(static_cast<E*>(a.dx) + row * a.ld_dx + at, o, K - at, a.vec_dx);
        }
    }
    if (!a.part) return;
    float* mine = a.part + int64_t(blockIdx.x) * a.K;
    if (a.threads <= 32) {                  // (V = 1) several rows at a time: the groups' shares first
#pragma unroll
        for (int i = 0; i < 4; ++i) split(dw[0][i], group_share[threadIdx.x * 8 + 2 * i], group_share[threadIdx.x * 8 + 2 * i + 1]);
        __syncthreads();
        for (int k = threadIdx.x; k < a.K; k += blockDim.x) {
            float s = 0.0f;
            for (int g = 0; g < per_cta; ++g) s += group_share[g * a.threads * 8 + k];
            mine[k] = s;
        }
        return;
    }
#pragma unroll
    for (int j = 0; j < V; ++j)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int k = (t + j * a.threads) * 8 + 2 * i;
            float even, odd;
            split(dw[j][i], even, odd);
            if (k < a.K) mine[k] = even;
            if (k + 1 < a.K) mine[k + 1] = odd;
        }
}

// dweight: 32 columns a CTA, eight warps over the shares (8192 FP32 additions a column at most).
template <int T>
__global__ void __launch_bounds__(256) dweight_kernel(const float* part, int shares, int K, void* dw, int f32) {
    __shared__ float s[8][32];
    after_previous();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, k = blockIdx.x * 32 + lane;
    float v = 0.0f;
    if (k < K)
        for (int g = warp; g < shares; g += 8) v += part[int64_t(g) * K + k];
    s[warp][lane] = v;
    __syncthreads();
    if (warp || k >= K) return;
#pragma unroll
    for (int i = 1; i < 8; ++i) v += s[i][lane];
    if (f32) static_cast<float*>(dw)[k] = v;
    else if constexpr (T == EF_F32) static_cast<float*>(dw)[k] = v;
    else if constexpr (T == EF_BF16) static_cast<__nv_bfloat16*>(dw)[k] = __float2bfloat16_rn(v);
    else static_cast<__half*>(dw)[k] = __float2half_rn(v);
}

struct BackShape { int threads, v; unsigned block; int64_t ctas; };
BackShape back_shape(int64_t M, int K) {
    const int eights = (K + 7) / 8;
    BackShape s;
    s.v = 1;
    if (eights <= 32) s.threads = eights <= 8 ? 8 : (eights <= 16 ? 16 : 32);
    else {
        while (eights > s.v * MAX_THREADS) s.v *= 2;
        s.threads = ((eights + s.v - 1) / s.v + 31) / 32 * 32;
    }
    s.block = s.threads > 32 ? unsigned(s.threads) : 128u;
    const int64_t per_cta = s.threads > 32 ? 1 : 128 / s.threads, want = (M + per_cta - 1) / per_cta, most = 148 * (1024 / s.block);
    s.ctas = want < most ? want : most;
    return s;
}
template <int T, bool VEC>
cudaError_t launch(const BackArgs& a, const BackShape& s, cudaStream_t stream) {
    const dim3 grid{unsigned(s.ctas)};
    switch (s.v) {
        case 1: return enqueue(backward_kernel<T, 1, true, VEC>, grid, s.block, 0, stream, a);
        case 2: return enqueue(backward_kernel<T, 2, true, VEC>, grid, s.block, 0, stream, a);
        case 4: return enqueue(backward_kernel<T, 4, T != EF_F32, VEC>, grid, s.block, 0, stream, a);
        default: return enqueue(backward_kernel<T, 8, false, VEC>, grid, s.block, 0, stream, a);
    }
}
template <int T>
cudaError_t launch(BackArgs a, const BackShape& s, void* dweight, cudaStream_t stream) {
    a.threads = s.threads;
    a.inverse_k = 1.0f / float(a.K);
    const bool vec = a.K % 8 == 0 && a.vec_dy && a.vec_h && a.vec_dx && a.vec_w && (!a.dres || a.vec_res);
    cudaError_t err = cudaSuccess;
    if (s.ctas) err = vec ? launch<T, true>(a, s, stream) : launch<T, false>(a, s, stream);
    if (err == cudaSuccess && dweight)
        err = enqueue(dweight_kernel<T>, dim3(unsigned((a.K + 31) / 32)), 256, 0, stream, a.part, int(s.ctas), a.K, dweight, a.w_f32);
    return err;
}
}  // namespace
}  // namespace rows

size_t rms_norm_backward_workspace(int64_t M, int64_t K) { return size_t(rows::back_shape(M, int(K)).ctas) * size_t(K) * 4; }

int launch_rms_norm_backward(int fmt, int64_t M, int64_t K, const mmasim_rms_norm_backward_args& p, cudaStream_t stream) {
    using namespace rows;
    const int bytes = fmt == EF_F32 ? 4 : 2;
    auto vec = [&](const void* q, int64_t ld, int size) { return int((reinterpret_cast<uintptr_t>(q) | uintptr_t(ld * size)) % 16 == 0); };
    BackArgs a = {};
    a.M = M; a.K = int(K);
    a.dy = p.dy; a.h = p.h; a.w = p.weight; a.dres = p.dresidual; a.dx = p.dx;
    a.part = p.dweight ? static_cast<float*>(p.workspace) : nullptr;
    a.ld_dy = p.ld_dy ? p.ld_dy : K; a.ld_h = p.ld_h ? p.ld_h : K; a.ld_res = p.ld_dresidual ? p.ld_dresidual : K; a.ld_dx = p.ld_dx ? p.ld_dx : K;
    a.eps = p.eps;
    a.w_f32 = p.weight_fmt == MMASIM_F32;
    a.vec_dy = vec(p.dy, a.ld_dy, bytes); a.vec_h = vec(p.h, a.ld_h, bytes); a.vec_res = vec(p.dresidual, a.ld_res, bytes); a.vec_dx = vec(p.dx, a.ld_dx, bytes);
    a.vec_w = vec(p.weight, 0, 4);
    const BackShape s = back_shape(M, int(K));
    const cudaError_t err = fmt == EF_F32 ? launch<EF_F32>(a, s, p.dweight, stream) : fmt == EF_BF16 ? launch<EF_BF16>(a, s, p.dweight, stream) : launch<EF_F16>(a, s, p.dweight, stream);
    if (err != cudaSuccess) { set_error("mmasim_rms_norm_backward: %s", cudaGetErrorString(err)); return MMASIM_ERR_CUDA; }
    return MMASIM_OK;
}

}  // namespace mmasim
