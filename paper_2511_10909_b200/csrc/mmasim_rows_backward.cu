// Gradients of the root-mean-square norm (mmasim_rms_norm_backward).  With r = 1 / sqrt(mean h^2 + eps) and g = dy w, by row:
//
//   dx = r (g - (h r) m) + dresidual,  m = (r / K) sum(g h)         dweight = sum over rows of dy (h r)
//
// (In this order no factor leaves FP32 that dx does not: h r is of size one, m of g's.  r^3, of which the formula is often written, is subnormal
// for rows from 4e12 on, zero from 1e15 on, and infinite for those below 1e-13 where eps is 0.)
// One pass: both sums of a row (h^2 and g h) come from the same loads, so nothing of the forward pass has to be kept but h.  Memory is what
// bounds it (8 bytes an element in BF16 with a residual).  A CTA walks over rows, a thread keeps its columns and with them its share of
// dweight in registers; the CTAs' shares go to the workspace, and a second kernel adds them column by column, in one order whatever runs first.
// The rows to come are on their way into shared memory meanwhile (asynchronous copies; a thread reads what it copied, so that no barrier but
// the sums' is needed).
#include "mmasim_quant.cuh"

namespace mmasim {
namespace rows {
namespace {
using namespace quant;

constexpr int MAX_THREADS = 512;
constexpr int SHORT_ROW = 128;              // eights

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

// The CTA's share of dweight; `group_share`: 32 bytes times V a thread of shared memory that nothing else uses any more, where rows are of a
// warp or less (then the shares of the CTA's groups are put together first).
template <int V, bool VEC, int PER = 1>
__device__ __forceinline__ void store_shares(const BackArgs& a, const Pair (&dw)[V][4], float* group_share, int per_cta, int t) {
    float* mine = a.part + int64_t(blockIdx.x) * a.K;
    const bool groups = a.threads <= 32;
    const int pitch = a.threads * 8 * V;
    float* to = groups ? group_share + threadIdx.x / a.threads * pitch : mine;
    const int K = groups ? pitch : a.K;
#pragma unroll
    for (int j = 0; j < V; ++j) {
        float v[8];
#pragma unroll
        for (int i = 0; i < 4; ++i) split(dw[j][i], v[2 * i], v[2 * i + 1]);
        if constexpr (VEC) {
            const int k = (t + j * PER * a.threads) * (8 / PER), next = PER == 1 ? 4 : a.threads * 4;
            if (k < K) *reinterpret_cast<float4*>(to + k) = make_float4(v[0], v[1], v[2], v[3]);
            if (k + next < K) *reinterpret_cast<float4*>(to + k + next) = make_float4(v[4], v[5], v[6], v[7]);
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const int k = t + (j * 8 + i) * a.threads;
                if (k < K) to[k] = v[i];
            }
        }
    }
    if (!groups) return;
    __syncthreads();
    for (int k = threadIdx.x; k < a.K; k += blockDim.x) {
        float sum = 0.0f;
        for (int g = 0; g < per_cta; ++g) sum += group_share[g * pitch + k];
        mine[k] = sum;
    }
}

extern __shared__ __align__(16) unsigned char back_smem[];

// HOLD: dy and h stay in registers between the sums and the results; else they are read again (rows too long for that).
template <int T, int V, bool HOLD, bool VEC>
__global__ void __launch_bounds__(MAX_THREADS) backward_kernel(const BackArgs a) {
    using E = typename Elem<T>::type;
    __shared__ float2 slots[2][16];
    after_previous();
    const int per_cta = a.threads > 32 ? 1 : int(blockDim.x) / a.threads;
    const int group = a.threads > 32 ? 0 : threadIdx.x / a.threads, t = a.threads > 32 ? threadIdx.x : threadIdx.x & (a.threads - 1);
    // (VEC: an eight side by side; else its elements a row's threads apart, neighbouring threads at neighbouring elements)
    auto place = [&](int j) { return VEC ? (t + j * a.threads) * 8 : t + j * 8 * a.threads; };
    auto load = [&](const E* p, int at, int K) {
        if constexpr (VEC) return load8<T, true>(p + at, K - at, true);
        else return load_spread<T>(p + at, K - at, a.threads);
    };
    auto weight = [&](int at, int K, Pair (&to)[4]) {
        if constexpr (VEC) load_weight8<T, true>(a.w, a.w_f32, at, K - at, true, to);
        else load_weight_spread<T>(a.w, a.w_f32, at, K - at, a.threads, to);
    };
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
                const int at = place(j);
                h_raw[j] = load(h, at, K);
                dy_raw[j] = load(dy, at, K);
                if (a.dres) res_raw[j] = load(static_cast<const E*>(a.dres) + row * a.ld_res, at, K);
            }
        }
        Pair squares = 0, products = 0;
#pragma unroll
        for (int j = 0; j < V; ++j) {
            const int at = place(j);
            if constexpr (!HOLD) {
                h_raw[0] = load(h, at, K);
                dy_raw[0] = load(dy, at, K);
            }
            Pair hv[4], g[4], w[4];
            widen<T>(h_raw[HOLD ? j : 0], hv);
            widen<T>(dy_raw[HOLD ? j : 0], g);
            weight(at, K, w);
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
        const Pair rr = both(r), m = both(-__fmul_rn(__fmul_rn(r, sums.y), a.inverse_k));
#pragma unroll
        for (int j = 0; j < V; ++j) {
            const int at = place(j);
            if (at >= K) continue;
            if constexpr (!HOLD) {
                h_raw[0] = load(h, at, K);
                dy_raw[0] = load(dy, at, K);
                if (a.dres) res_raw[0] = load(static_cast<const E*>(a.dres) + row * a.ld_res, at, K);
            }
            Pair hv[4], g[4], w[4], out[4];
            widen<T>(h_raw[HOLD ? j : 0], hv);
            widen<T>(dy_raw[HOLD ? j : 0], g);
            weight(at, K, w);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const Pair unit = mul2(hv[i], rr);
                dw[j][i] = fma2(g[i], unit, dw[j][i]);
                out[i] = mul2(fma2(unit, m, mul2(g[i], w[i])), rr);
            }
            if (a.dres) {
                Pair res[4];
                widen<T>(res_raw[HOLD ? j : 0], res);
#pragma unroll
                for (int i = 0; i < 4; ++i) out[i] = add2(out[i], res[i]);
            }
            Raw<T> o;
            narrow<T>(out, o);
            if constexpr (VEC) store8<T, true>(static_cast<E*>(a.dx) + row * a.ld_dx + at, o, 8, true);
            else store_spread<T>(static_cast<E*>(a.dx) + row * a.ld_dx + at, o, K - at, a.threads);
        }
    }
    if (a.part) store_shares<V, VEC>(a, dw, reinterpret_cast<float*>(back_smem), per_cta, t);
}

// Both sums of the row's threads with half the exchanges: after the first, one half of a warp has one sum and the other the other.
// `slot`: 32 words of shared memory that nothing else uses.
__device__ __forceinline__ float2 row_sums_wide(float2 v, int threads, float* slot) {
    const int lane = threadIdx.x & 31;
    const bool upper = lane >= 16;
    float s = (upper ? v.y : v.x) + __shfl_xor_sync(0xFFFFFFFFu, upper ? v.x : v.y, 16);
#pragma unroll
    for (int o = 8; o > 0; o >>= 1) s += __shfl_xor_sync(0xFFFFFFFFu, s, o);
    if (threads > 32) {
        if ((lane & 15) == 0) slot[lane + (threadIdx.x >> 5)] = s;
        __syncthreads();
        s = (lane & 15) < threads / 32 ? slot[lane] : 0.0f;
#pragma unroll
        for (int o = 8; o > 0; o >>= 1) s += __shfl_xor_sync(0xFFFFFFFFu, s, o);
    }
    return make_float2(__shfl_sync(0xFFFFFFFFu, s, 0), __shfl_sync(0xFFFFFFFFu, s, 16));
}

// The same for whole eights at multiples of 16 bytes: `depth` rows (2 or 3) of h, dy and dresidual in shared memory, the threads' slots of 16
// bytes side by side (a thread's own side by side, free of conflicts between banks too: 4096 x 4096 45 us instead of 34).
template <int T, int V> constexpr int RING_SLOTS = 3 * V * (Elem<T>::WORDS / 4);
template <int T, int V>
__global__ void __launch_bounds__(MAX_THREADS) backward_ring_kernel(const BackArgs a, const int depth) {
    using E = typename Elem<T>::type;
    // slots of an eight, elements of a slot; slots lie a row's threads apart, so that neighbouring threads copy and store neighbouring 16 bytes
    // (an FP32 eight in one piece: half of every sector at a time, 4096 x 4096 68.8 us instead of 47.0)
    constexpr int PER = Elem<T>::WORDS / 4, EACH = 16 / sizeof(E);
    __shared__ float slots[2][32];
    after_previous();
    const int per_cta = a.threads > 32 ? 1 : int(blockDim.x) / a.threads;
    const int group = a.threads > 32 ? 0 : threadIdx.x / a.threads, t = a.threads > 32 ? threadIdx.x : threadIdx.x & (a.threads - 1);
    const int64_t stride = int64_t(gridDim.x) * per_cta;
    const uint32_t plane = blockDim.x * 16, stage = plane * RING_SLOTS<T, V>, mine = threadIdx.x * 16, end = mine + depth * stage;
    uint32_t in = mine, out = mine;                     // of the row to be fetched and to be read next
    int64_t ahead = int64_t(blockIdx.x) * per_cta + group;
    const E *dy = static_cast<const E*>(a.dy) + ahead * a.ld_dy + t * EACH, *h_at = static_cast<const E*>(a.h) + ahead * a.ld_h + t * EACH;
    const E* res_at = a.dres ? static_cast<const E*>(a.dres) + ahead * a.ld_res + t * EACH : nullptr;
    E* dx = static_cast<E*>(a.dx) + ahead * a.ld_dx + t * EACH;
    auto fetch = [&]() {
        if (ahead < a.M) {
            const uint32_t to = uint32_t(__cvta_generic_to_shared(back_smem)) + in;
#pragma unroll
            for (int slot = 0; slot < V * PER; ++slot) {
                const int at = slot * a.threads * EACH;
                if (at + t * EACH >= a.K) continue;
                asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" :: "r"(to + slot * plane), "l"(h_at + at) : "memory");
                asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" :: "r"(to + (V * PER + slot) * plane), "l"(dy + at) : "memory");
                if (a.dres) asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" :: "r"(to + (2 * V * PER + slot) * plane), "l"(res_at + at) : "memory");
            }
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
        in = in + stage == end ? mine : in + stage;
        ahead += stride;
        h_at += stride * a.ld_h;
        dy += stride * a.ld_dy;
        res_at += stride * a.ld_res;
    };
    for (int i = 1; i < depth; ++i) fetch();

    Pair w[V][4], dw[V][4];
#pragma unroll
    for (int j = 0; j < V; ++j) {
        if constexpr (PER == 1) {
            const int at = (t + j * a.threads) * 8;
            load_weight8<T, true>(a.w, a.w_f32, at, a.K - at, true, w[j]);
        } else {
#pragma unroll
            for (int i = 0; i < PER; ++i) {
                const int at = ((j * PER + i) * a.threads + t) * EACH;
                const float4 q = a.w && at < a.K ? *reinterpret_cast<const float4*>(static_cast<const float*>(a.w) + at) : make_float4(1.0f, 1.0f, 1.0f, 1.0f);
                w[j][2 * i] = pair(q.x, q.y);
                w[j][2 * i + 1] = pair(q.z, q.w);
            }
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) dw[j][i] = 0;
    }
    int turn = 0;
    for (int64_t first = int64_t(blockIdx.x) * per_cta; first < a.M; first += stride, turn ^= 1) {
        const int K = first + group < a.M ? a.K : 0;
        fetch();
        if (depth == 3) asm volatile("cp.async.wait_group 2;" ::: "memory");
        else asm volatile("cp.async.wait_group 1;" ::: "memory");
        auto there = [&](int slot) { return (slot * a.threads + t) * EACH < K; };
        auto take = [&](int which, int j) {             // (zeros where there is nothing)
            Raw<T> r;
#pragma unroll
            for (int i = 0; i < PER; ++i) {
                uint4 q = make_uint4(0, 0, 0, 0);
                if (PER == 1 || there(j * PER + i)) q = *reinterpret_cast<const uint4*>(back_smem + out + ((which * V + j) * PER + i) * plane);
                r.w[4 * i] = q.x; r.w[4 * i + 1] = q.y; r.w[4 * i + 2] = q.z; r.w[4 * i + 3] = q.w;
            }
            return r;
        };
        Pair squares = 0, products = 0;
#pragma unroll
        for (int j = 0; j < V; ++j) {
            if (!there(j * PER)) continue;
            Pair hv[4], gv[4];
            widen<T>(take(0, j), hv);
            widen<T>(take(1, j), gv);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                squares = fma2(hv[i], hv[i], squares);
                products = fma2(mul2(gv[i], w[j][i]), hv[i], products);
            }
        }
        float2 sums, odd;
        split(squares, sums.x, odd.x);
        split(products, sums.y, odd.y);
        sums = make_float2(sums.x + odd.x, sums.y + odd.y);
        sums = a.threads >= 32 ? row_sums_wide(sums, a.threads, slots[turn]) : row_sums(sums, a.threads, nullptr);       // (two sets of slots: one barrier a row)
        const float r = inverse_root(__fmaf_rn(sums.x, a.inverse_k, a.eps));
        const Pair rr = both(r), m = both(-__fmul_rn(__fmul_rn(r, sums.y), a.inverse_k));
#pragma unroll
        for (int j = 0; j < V; ++j) {
            if (!there(j * PER)) continue;
            Pair hv[4], gv[4], o[4];        // (read again: held, their registers cost CTAs their place, 4096 x 4096 43 us instead of 34)
            widen<T>(take(0, j), hv);
            widen<T>(take(1, j), gv);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const Pair unit = mul2(hv[i], rr);
                dw[j][i] = fma2(gv[i], unit, dw[j][i]);
                o[i] = mul2(fma2(unit, m, mul2(gv[i], w[j][i])), rr);
            }
            if (a.dres) {
                Pair res[4];
                widen<T>(take(2, j), res);
#pragma unroll
                for (int i = 0; i < 4; ++i) o[i] = add2(o[i], res[i]);
            }
            Raw<T> raw;
            narrow<T>(o, raw);
#pragma unroll
            for (int i = 0; i < PER; ++i)
                if (there(j * PER + i))
                    *reinterpret_cast<uint4*>(dx + (j * PER + i) * a.threads * EACH) = make_uint4(raw.w[4 * i], raw.w[4 * i + 1], raw.w[4 * i + 2], raw.w[4 * i + 3]);
        }
        out = out + stage == end ? mine : out + stage;
        dx += stride * a.ld_dx;
    }
    if (!a.part) return;
    asm volatile("cp.async.wait_all;" ::: "memory");
    __syncthreads();
    store_shares<V, true, PER>(a, dw, reinterpret_cast<float*>(back_smem), per_cta, t);
}

// dweight: COLS columns a CTA, 1024 / COLS threads over the shares of each.
template <int T, int COLS>
__global__ void __launch_bounds__(1024) dweight_kernel(const float* part, int shares, int K, void* dw, int f32) {
    constexpr int PARTS = 1024 / COLS;
    __shared__ float s[32][COLS];
    after_previous();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, col = lane % COLS, k = blockIdx.x * COLS + col;
    float v = 0.0f;
    if (k < K) {
        for (int g = threadIdx.x / COLS; g < shares; g += PARTS * 8) {
            float p[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) p[i] = g + PARTS * i < shares ? part[int64_t(g + PARTS * i) * K + k] : 0.0f;
#pragma unroll
            for (int i = 0; i < 8; ++i) v += p[i];
        }
    }
    auto columns = [&]() {                  // over a warp's lanes of the same column
#pragma unroll
        for (int o = COLS; o < 32; o *= 2) v += __shfl_xor_sync(0xFFFFFFFFu, v, o);
    };
    columns();
    if (lane < COLS) s[warp][lane] = v;
    __syncthreads();
    if (warp) return;
    v = 0.0f;
#pragma unroll
    for (int i = 0; i < COLS; ++i) v += s[lane / COLS * COLS + i][col];
    columns();
    if (lane >= COLS || k >= K) return;
    if (f32) static_cast<float*>(dw)[k] = v;
    else if constexpr (T == EF_F32) static_cast<float*>(dw)[k] = v;
    else if constexpr (T == EF_BF16) static_cast<__nv_bfloat16*>(dw)[k] = __float2bfloat16_rn(v);
    else static_cast<__half*>(dw)[k] = __float2half_rn(v);
}

// Threads per row, eights per thread, CTAs: what the workspace goes by too, so by sizes alone (whether the call takes the ring or not).
struct BackShape { int threads, v; unsigned block; int64_t ctas; };
BackShape back_shape(int64_t M, int K) {
    const int eights = (K + 7) / 8;
    BackShape s;
    s.v = 1;
    if (K % 8 == 0 && eights <= SHORT_ROW)
        while (s.v < 4 && eights > s.v * 8 && M * eights >= 2 * s.v * 148 * 256) s.v *= 2;
    const int threads = (eights + s.v - 1) / s.v;
    if (threads <= 32) s.threads = threads <= 8 ? 8 : (threads <= 16 ? 16 : 32);
    else {
        s.v = 1;
        while (s.v < 4 && eights > s.v * 256) s.v *= 2;
        while (eights > s.v * MAX_THREADS) s.v *= 2;
        s.threads = ((eights + s.v - 1) / s.v + 31) / 32 * 32;
    }
    s.block = s.threads > 32 ? unsigned(s.threads) : 128u;
    // as many as an SM holds with their rings and registers (BF16 with a residual, CTAs an SM 2 / 3 / 4: 4096 x 4096 32.6 / 41.0 / 36.8 us,
    // 16384 x 8192 174 / 207 / 183; one eight a thread, 16384 x 1024 46.9 / 37.9 / 34.2), but two rows each: their shares are read again
    const int64_t per_cta = s.threads > 32 ? 1 : 128 / s.threads, want = (M + per_cta - 1) / per_cta, few = (want + 1) / 2 < 148 ? 148 : (want + 1) / 2;
    int64_t most = 148 * (s.v > 1 && s.threads > 32 ? 2 : 4);
    if (most > few) most = few;
    s.ctas = want < most ? want : most;
    return s;
}
constexpr size_t RING_MOST = 216 * 1024;
template <int T, int V>
cudaError_t launch_ring(const BackArgs& a, const BackShape& s, cudaStream_t stream) {
    const size_t row = size_t(RING_SLOTS<T, V>) * 16 * s.block;
    const int depth = 3 * row * (s.ctas / 148 > 1 ? size_t(s.ctas / 148) : 1) <= RING_MOST ? 3 : 2;
    const size_t smem = depth * row;
    if (smem > 40 * 1024) {                 // (the sums' slots and the groups' shares come on top)
        const cudaError_t err = cudaFuncSetAttribute(backward_ring_kernel<T, V>, cudaFuncAttributeMaxDynamicSharedMemorySize, int(RING_MOST));
        if (err != cudaSuccess) { cudaGetLastError(); return err; }
    }
    return enqueue(backward_ring_kernel<T, V>, dim3(unsigned(s.ctas)), s.block, smem, stream, a, depth);
}
constexpr size_t two_rows(int words, int v, unsigned block) { return size_t(2) * 3 * v * (words / 4) * 16 * block; }       // of the ring
template <int T, bool VEC>
cudaError_t launch(const BackArgs& a, const BackShape& s, cudaStream_t stream) {
    const dim3 grid{unsigned(s.ctas)};
    if constexpr (VEC) {
        constexpr int WORDS = Elem<T>::WORDS;
        static_assert(two_rows(WORDS, 2, MAX_THREADS) <= RING_MOST && (T == EF_F32 || two_rows(WORDS, 4, MAX_THREADS) <= RING_MOST),
                      "the ring holds two rows of all threads but of four eights each in FP32, and of eight");
        if (s.v == 1) return launch_ring<T, 1>(a, s, stream);
        if (s.v == 2) return launch_ring<T, 2>(a, s, stream);
        if (s.v == 4) {
            if constexpr (T == EF_F32)
                if (two_rows(WORDS, 4, s.block) > RING_MOST) return enqueue(backward_kernel<T, 4, false, true>, grid, s.block, 0, stream, a);
            return launch_ring<T, 4>(a, s, stream);
        }
        return enqueue(backward_kernel<T, 8, false, true>, grid, s.block, 0, stream, a);
    } else {
        const size_t share = s.threads > 32 ? 0 : size_t(32) * s.v * s.block;
        switch (s.v) {
            case 1: return enqueue(backward_kernel<T, 1, true, false>, grid, s.block, share, stream, a);
            case 2: return enqueue(backward_kernel<T, 2, true, false>, grid, s.block, share, stream, a);
            case 4: return enqueue(backward_kernel<T, 4, T != EF_F32, false>, grid, s.block, share, stream, a);
            default: return enqueue(backward_kernel<T, 8, false, false>, grid, s.block, 0, stream, a);
        }
    }
}
template <int T>
cudaError_t launch(BackArgs a, BackShape s, void* dweight, cudaStream_t stream) {
    a.threads = s.threads;
    a.inverse_k = 1.0f / float(a.K);
    const bool vec = a.K % 8 == 0 && a.vec_dy && a.vec_h && a.vec_dx && a.vec_w && (!a.dres || a.vec_res);
    if (vec) {                              // no more than have room for two rows of the ring
        const int64_t room = int64_t(RING_MOST / two_rows(Elem<T>::WORDS, s.v, s.block));
        if (room && s.ctas > 148 * room) s.ctas = 148 * room;
    }
    cudaError_t err = cudaSuccess;
    if (s.ctas) err = vec ? launch<T, true>(a, s, stream) : launch<T, false>(a, s, stream);
    if (err == cudaSuccess && dweight) {    // columns a CTA by whether the CTAs of 8 have room at once (us with 8 / 32: K = 128 15.9 / 17.0, 2048 32.2 / 32.8, 4096 34.4 / 32.6)
        const bool few = a.K <= 8 * 2 * 148;
        err = few ? enqueue(dweight_kernel<T, 8>, dim3(unsigned((a.K + 7) / 8)), 1024, 0, stream, a.part, int(s.ctas), a.K, dweight, a.w_f32)
                  : enqueue(dweight_kernel<T, 32>, dim3(unsigned((a.K + 31) / 32)), 1024, 0, stream, a.part, int(s.ctas), a.K, dweight, a.w_f32);
    }
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
