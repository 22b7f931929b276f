// layernorm.cu -- LayerNorm over the rows of x [T, d] and its backward pass, for model
// families whose blocks normalise with the mean removed.
//
//   forward   mu = mean_j x_j, sigma = sqrt(mean_j (x_j - mu)^2 + eps)
//             y = gamma (.) (x - mu) / sigma + beta
//   backward  xhat = (x - mu) / sigma, u = gamma (.) g
//             g_out = (u - mean(u) - xhat mean(u (.) xhat)) / max(sigma, min_rms)
//             dgamma = sum_t g_t (.) xhat_t,  dbeta = sum_t g_t
//
// Rows of up to 8192 elements stay in a block's registers and are read once: the variance is
// the sum of squares around the row's own mean (a difference of two large sums would lose it),
// and the backward pass forms mu and sigma again from the row that it has to read anyway, so no
// statistics are saved between the passes.  A row's next vectors are loaded before the
// reductions of the one at hand.  Each thread keeps the same columns for every row of its
// block, so the weight sums stay in its registers until the last row; the blocks' sums are then
// added in block order by a second kernel, or in a short batch within its one cluster (no
// atomics: repeat calls give identical bits).  Longer rows go through the row in several passes, and their weight
// sums through a kernel of their own.
//
// Bound: HBM.
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <math.h>

#include "internal.h"
#include "ptx.cuh"

namespace fpo {
namespace {

// One vector of a row: 16 bytes, or 1 element where rows are not 16-byte aligned.
template <typename TT, int VEC>
struct RowVec;
template <>
struct RowVec<__nv_bfloat16, 8> {
    uint4 r;
    __device__ __forceinline__ void zero() { r = make_uint4(0u, 0u, 0u, 0u); }
    __device__ __forceinline__ void load(const __nv_bfloat16* p) {
        r = *reinterpret_cast<const uint4*>(p);
    }
    __device__ __forceinline__ void get(float (&v)[8]) const {
        const uint32_t w[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            v[2 * k] = __uint_as_float(w[k] << 16);
            v[2 * k + 1] = __uint_as_float(w[k] & 0xffff0000u);
        }
    }
    static __device__ __forceinline__ void store(__nv_bfloat16* p, const float (&v)[8]) {
        uint4 a;
        __nv_bfloat162* h = reinterpret_cast<__nv_bfloat162*>(&a);
#pragma unroll
        for (int k = 0; k < 4; ++k) h[k] = __floats2bfloat162_rn(v[2 * k], v[2 * k + 1]);
        *reinterpret_cast<uint4*>(p) = a;
    }
};
template <>
struct RowVec<float, 4> {
    float4 r;
    __device__ __forceinline__ void zero() { r = make_float4(0.f, 0.f, 0.f, 0.f); }
    __device__ __forceinline__ void load(const float* p) { r = *reinterpret_cast<const float4*>(p); }
    __device__ __forceinline__ void get(float (&v)[4]) const {
        v[0] = r.x;
        v[1] = r.y;
        v[2] = r.z;
        v[3] = r.w;
    }
    static __device__ __forceinline__ void store(float* p, const float (&v)[4]) {
        *reinterpret_cast<float4*>(p) = make_float4(v[0], v[1], v[2], v[3]);
    }
};
template <>
struct RowVec<float, 1> {
    float r;
    __device__ __forceinline__ void zero() { r = 0.f; }
    __device__ __forceinline__ void load(const float* p) { r = *p; }
    __device__ __forceinline__ void get(float (&v)[1]) const { v[0] = r; }
    static __device__ __forceinline__ void store(float* p, const float (&v)[1]) { *p = v[0]; }
};

// Sums of N values over the W warps that share a row, the same bits in every thread: a
// butterfly per warp, then one over the warps' sums, which every warp reads one to a lane (all
// threads adding all W of them took 0.6 us a row with 16 warps).  `at` alternates between two
// areas from call to call, so one barrier a call is enough.
template <int N, int W>
struct RowSum {
    float (*sh)[2][N][W];  // shared (W > 1 only), this row group's
    int group;             // of the block's row groups
    int at;
    __device__ __forceinline__ void operator()(float (&v)[N]) {
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) {
#pragma unroll
            for (int k = 0; k < N; ++k) v[k] += __shfl_xor_sync(0xffffffffu, v[k], o);
        }
        if constexpr (W > 1) {
            const int w = (threadIdx.x >> 5) % W, lane = threadIdx.x & 31;
            if (lane == 0) {
#pragma unroll
                for (int k = 0; k < N; ++k) (*sh)[at][k][w] = v[k];
            }
            __syncwarp();
            // the row group's own barrier (0 is __syncthreads)
            asm volatile("bar.sync %0, %1;" ::"r"(group + 1), "n"(32 * W) : "memory");
#pragma unroll
            for (int k = 0; k < N; ++k) v[k] = (*sh)[at][k][lane % W];
#pragma unroll
            for (int o = W / 2; o > 0; o >>= 1) {
#pragma unroll
                for (int k = 0; k < N; ++k) v[k] += __shfl_xor_sync(0xffffffffu, v[k], o);
            }
            at ^= 1;
        }
    }
};

// TH threads to a row, blocks of 256 threads (512 for the longest rows) with 256 / TH rows at a
// time, NV vectors of VEC elements per thread: vector v of thread t of a row holds elements
// (v TH + t) VEC ...
template <int TH>
constexpr int ln_threads() {
    return TH == 512 ? 512 : 256;
}
template <int TH>
constexpr int ln_rows() {
    return ln_threads<TH>() / TH;
}
// Elements of a row per thread, at most; twice that for the longest fp32 rows.
template <typename TT, int TH = 256>
constexpr int ln_ept() {
    return sizeof(TT) == 2 || TH == 512 ? 16 : 8;
}
// Blocks per SM that the registers have to leave room for.
template <int TH, bool kBack>
constexpr int ln_min_blocks() {
    return TH == 512 ? 1 : kBack ? 2 : 3;
}

// A thread's vectors of a row, and their elements in pairs for packed arithmetic (a last odd
// one with a zero).  The number of instructions bounds the passes over a row as much as its
// bytes do: with scalar arithmetic and the weights read again in every pass the backward
// pass of T 16384, d 4096 took 124 us.
template <typename TT, int VEC, int NV, int TH>
struct RowPart {
    static constexpr int kE = VEC * NV, kPairs = (kE + 1) / 2;
    using V = RowVec<TT, VEC>;
    V r[NV];
    // (outside the row: zeros)
    __device__ __forceinline__ void load(const TT* p, int t, int d) {
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            const int k = (v * TH + t) * VEC;
            if (k < d)
                r[v].load(p + k);
            else
                r[v].zero();
        }
    }
    __device__ __forceinline__ void get(float2 (&f)[kPairs]) const {
        float e[2 * kPairs];
        if constexpr (kE % 2) e[kE] = 0.f;
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            float x[VEC];
            r[v].get(x);
#pragma unroll
            for (int q = 0; q < VEC; ++q) e[v * VEC + q] = x[q];
        }
#pragma unroll
        for (int i = 0; i < kPairs; ++i) f[i] = make_float2(e[2 * i], e[2 * i + 1]);
    }
    static __device__ __forceinline__ void store(TT* p, int t, int d, const float2 (&f)[kPairs]) {
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            const int k = (v * TH + t) * VEC;
            float x[VEC];
#pragma unroll
            for (int q = 0; q < VEC; ++q) {
                const float2& w = f[(v * VEC + q) / 2];
                x[q] = (v * VEC + q) % 2 ? w.y : w.x;
            }
            if (k < d) V::store(p + k, x);
        }
    }
    // Whether element e of the thread's is inside the row.
    static __device__ __forceinline__ bool in(int e, int t, int d) {
        return e < kE && (e / VEC * TH + t) * VEC < d;
    }
};

__device__ __forceinline__ float2 both(float a) { return make_float2(a, a); }

// x - mu, zero outside the row.
template <class P, int TH>
__device__ __forceinline__ void center(float2 (&x)[P::kPairs], float mu, int t, int d, bool full) {
    const float2 m = both(-mu);
#pragma unroll
    for (int i = 0; i < P::kPairs; ++i) x[i] = __fadd2_rn(x[i], m);
    if (full) return;
#pragma unroll
    for (int i = 0; i < P::kPairs; ++i) {
        if (!P::in(2 * i, t, d)) x[i].x = 0.f;
        if (!P::in(2 * i + 1, t, d)) x[i].y = 0.f;
    }
}

template <typename TT, int VEC, int NV, int TH>
__global__ void __launch_bounds__(ln_threads<TH>(), ln_min_blocks<TH, false>())
    layernorm_fwd_kernel(const TT* __restrict__ x, const TT* __restrict__ gamma,
                         const TT* __restrict__ beta, int T, int d, float eps,
                         TT* __restrict__ y, float* __restrict__ mean_out,
                         float* __restrict__ rstd_out) {
    using P = RowPart<TT, VEC, NV, TH>;
    constexpr int kW = TH / 32;
    __shared__ float sh[ln_rows<TH>()][2][1][kW];
    const int group = threadIdx.x / TH;
    RowSum<1, kW> row_sum{&sh[group], group, 0};
    const int t = threadIdx.x % TH;
    const float inv_d = 1.f / static_cast<float>(d);
    const bool full = d == TH * NV * VEC && P::kE % 2 == 0;  // every thread's elements inside
    P nx, w, b;
    if (gamma) w.load(gamma, t, d);
    if (beta) b.load(beta, t, d);
    const long long step = gridDim.x * ln_rows<TH>();
    long long row = blockIdx.x * ln_rows<TH>() + group;
    if (row < T) nx.load(x + row * d, t, d);
    for (; row < T; row += step) {
        float2 c[P::kPairs];
        float2 a = both(0.f);
        nx.get(c);
#pragma unroll
        for (int i = 0; i < P::kPairs; ++i) a = __fadd2_rn(a, c[i]);
        if (row + step < T) nx.load(x + (row + step) * d, t, d);
        float s[1] = {a.x + a.y};
        row_sum(s);
        const float mu = s[0] * inv_d;
        center<P, TH>(c, mu, t, d, full);
        a = both(0.f);
#pragma unroll
        for (int i = 0; i < P::kPairs; ++i) a = __ffma2_rn(c[i], c[i], a);
        s[0] = a.x + a.y;
        row_sum(s);
        const float rstd = 1.f / sqrtf(fmaf(s[0], inv_d, eps));
        float2 wf[P::kPairs], bf[P::kPairs];
        if (gamma) w.get(wf);
        if (beta) b.get(bf);
#pragma unroll
        for (int i = 0; i < P::kPairs; ++i) {
            c[i] = __fmul2_rn(c[i], both(rstd));
            if (gamma && beta)
                c[i] = __ffma2_rn(c[i], wf[i], bf[i]);
            else if (gamma)
                c[i] = __fmul2_rn(c[i], wf[i]);
            else if (beta)
                c[i] = __fadd2_rn(c[i], bf[i]);
        }
        P::store(y + row * d, t, d, c);
        if (t == 0) {
            if (mean_out) mean_out[row] = mu;
            if (rstd_out) rstd_out[row] = rstd;
        }
    }
}

// What becomes of the sums of g xhat and of g:
//   kPartSums     every block's to part[grid][2][d]; layernorm_cols_final_kernel adds them
//   kClusterSums  the grid is one cluster, whose blocks add each other's from shared memory, in
//                 block order, and write dgamma and dbeta: one launch and no workspace
enum LnSums { kNoSums = 0, kPartSums = 1, kClusterSums = 2 };
constexpr int kLnCluster = 8;

template <typename TT, int VEC, int NV, int TH, int kMode>
__global__ void __launch_bounds__(ln_threads<TH>(), ln_min_blocks<TH, true>())
    layernorm_vjp_kernel(const TT* __restrict__ g, const TT* __restrict__ x,
                         const TT* __restrict__ gamma, int T, int d, float eps, float min_rms,
                         TT* __restrict__ out, float* __restrict__ part,
                         float* __restrict__ dgamma, float* __restrict__ dbeta) {
    using P = RowPart<TT, VEC, NV, TH>;
    constexpr bool kSums = kMode != kNoSums;
    constexpr int kPairs = P::kPairs, kW = TH / 32;
    __shared__ float sh[ln_rows<TH>()][2][2][kW];
    const int group = threadIdx.x / TH;
    RowSum<2, kW> row_sum{&sh[group], group, 0};
    grid_dependency_trigger();
    const int t = threadIdx.x % TH;
    const float inv_d = 1.f / static_cast<float>(d);
    const bool full = d == TH * NV * VEC && P::kE % 2 == 0;
    P nx, ng, w;
    if (gamma) w.load(gamma, t, d);
    float2 dg[kSums ? kPairs : 1], db[kSums ? kPairs : 1];
#pragma unroll
    for (int i = 0; i < (kSums ? kPairs : 1); ++i) dg[i] = db[i] = both(0.f);
    const long long step = gridDim.x * ln_rows<TH>();
    long long row = blockIdx.x * ln_rows<TH>() + group;
    if (row < T) {
        nx.load(x + row * d, t, d);
        ng.load(g + row * d, t, d);
    }
    for (; row < T; row += step) {
        float2 c[kPairs], gv[kPairs], u[kPairs];
        float2 a0 = both(0.f), a1 = both(0.f);  // sums of x and of u = gamma g
        nx.get(c);
        ng.get(gv);
        if (gamma) {
            float2 wf[kPairs];
            w.get(wf);
#pragma unroll
            for (int i = 0; i < kPairs; ++i) u[i] = __fmul2_rn(gv[i], wf[i]);
        } else {
#pragma unroll
            for (int i = 0; i < kPairs; ++i) u[i] = gv[i];
        }
#pragma unroll
        for (int i = 0; i < kPairs; ++i) {
            a0 = __fadd2_rn(a0, c[i]);
            a1 = __fadd2_rn(a1, u[i]);
        }
        if (row + step < T) {
            nx.load(x + (row + step) * d, t, d);
            ng.load(g + (row + step) * d, t, d);
        }
        float s[2] = {a0.x + a0.y, a1.x + a1.y};
        row_sum(s);
        const float mu = __fmul_rn(s[0], inv_d), um = __fmul_rn(s[1], inv_d);
        center<P, TH>(c, mu, t, d, full);
        a0 = a1 = both(0.f);  // sums of (x - mu)^2 and of u (x - mu)
#pragma unroll
        for (int i = 0; i < kPairs; ++i) {
            a0 = __ffma2_rn(c[i], c[i], a0);
            a1 = __ffma2_rn(u[i], c[i], a1);
        }
        s[0] = a0.x + a0.y;
        s[1] = a1.x + a1.y;
        row_sum(s);
        const float sigma = sqrtf(fmaf(s[0], inv_d, eps));
        const float rstd = 1.f / sigma;
        const float cm = __fmul_rn(__fmul_rn(s[1], inv_d), rstd);  // mean(u xhat)
        const float2 pref = both(1.f / fmaxf(sigma, min_rms)), r2 = both(rstd), nc = both(-cm),
                     nu = both(-um);
#pragma unroll
        for (int i = 0; i < kPairs; ++i) {
            c[i] = __fmul2_rn(c[i], r2);  // xhat
            if constexpr (kSums) {
                dg[i] = __ffma2_rn(gv[i], c[i], dg[i]);
                db[i] = __fadd2_rn(db[i], gv[i]);
            }
            u[i] = __fmul2_rn(__ffma2_rn(c[i], nc, __fadd2_rn(u[i], nu)), pref);
        }
        if (out) P::store(out + row * d, t, d, u);
    }
    if constexpr (kSums) {
        constexpr int kCols = NV * TH * VEC;
        __shared__ float tot[kMode == kClusterSums ? 2 * kCols : 1];
        float* p = kMode == kClusterSums ? tot : part + static_cast<size_t>(blockIdx.x) * 2 * d;
        if constexpr (ln_rows<TH>() > 1) {
            // the block's row groups hold the same columns: their sums in group order
            __shared__ float acc[ln_rows<TH>()][kCols];
#pragma unroll
            for (int which = 0; which < 2; ++which) {
                __syncthreads();
#pragma unroll
                for (int e = 0; e < P::kE; ++e) {
                    const float2& f = which ? db[e / 2] : dg[e / 2];
                    acc[group][(e / VEC * TH + t) * VEC + e % VEC] = e % 2 ? f.y : f.x;
                }
                __syncthreads();
                for (int k = threadIdx.x; k < d; k += ln_threads<TH>()) {
                    float a = 0.f;
#pragma unroll
                    for (int r = 0; r < ln_rows<TH>(); ++r) a += acc[r][k];
                    p[which * d + k] = a;
                }
            }
        } else {
            float2 z[kPairs];
#pragma unroll
            for (int which = 0; which < 2; ++which) {
#pragma unroll
                for (int i = 0; i < kPairs; ++i) z[i] = which ? db[i] : dg[i];
#pragma unroll
                for (int e = 0; e < P::kE; ++e)
                    if (P::in(e, t, d))
                        p[which * d + (e / VEC * TH + t) * VEC + e % VEC] = e % 2 ? z[e / 2].y
                                                                                : z[e / 2].x;
            }
        }
        if constexpr (kMode == kClusterSums) {
            __syncwarp();
            cluster_sync();
            for (int k = blockIdx.x * ln_threads<TH>() + threadIdx.x; k < 2 * d;
                 k += kLnCluster * ln_threads<TH>()) {
                const uint32_t at = smem_u32(tot + k);
                float a = 0.f;
#pragma unroll
                for (int r = 0; r < kLnCluster; ++r)
                    a += __uint_as_float(ld_shared_cluster_u32(mapa_shared(at, r)));
                float* dst = k < d ? dgamma : dbeta;
                if (dst) dst[k < d ? k : k - d] = a;
            }
            __syncwarp();
            cluster_sync();  // until every block has read this one's
        }
    }
}

// ------------------------------------------------------------------ long rows
constexpr int kLongThreads = 512;

// mu and sigma of one row by the whole block, in two passes over it.
template <typename TT, int VEC>
__device__ __forceinline__ float2 long_stats(const TT* xr, int d, float eps,
                                             RowSum<2, kLongThreads / 32>& sum) {
    using V = RowVec<TT, VEC>;
    const float inv_d = 1.f / static_cast<float>(d);
    float s[2] = {0.f, 0.f};
    for (int k = threadIdx.x * VEC; k < d; k += kLongThreads * VEC) {
        float c[VEC];
        V v;
        v.load(xr + k);
        v.get(c);
#pragma unroll
        for (int q = 0; q < VEC; ++q) s[0] += c[q];
    }
    sum(s);
    const float mu = __fmul_rn(s[0], inv_d);
    s[0] = s[1] = 0.f;
    for (int k = threadIdx.x * VEC; k < d; k += kLongThreads * VEC) {
        float c[VEC];
        V v;
        v.load(xr + k);
        v.get(c);
#pragma unroll
        for (int q = 0; q < VEC; ++q) s[0] = fmaf(c[q] - mu, c[q] - mu, s[0]);
    }
    sum(s);
    return make_float2(mu, sqrtf(fmaf(s[0], inv_d, eps)));
}

template <typename TT, int VEC>
__global__ void __launch_bounds__(kLongThreads)
    layernorm_fwd_long_kernel(const TT* __restrict__ x, const TT* __restrict__ gamma,
                              const TT* __restrict__ beta, int T, int d, float eps,
                              TT* __restrict__ y, float* __restrict__ mean_out,
                              float* __restrict__ rstd_out) {
    using V = RowVec<TT, VEC>;
    __shared__ float sh[2][2][kLongThreads / 32];
    RowSum<2, kLongThreads / 32> sum{&sh, 0, 0};
    for (long long row = blockIdx.x; row < T; row += gridDim.x) {
        const TT* xr = x + row * d;
        const float2 st = long_stats<TT, VEC>(xr, d, eps, sum);
        const float rstd = 1.f / st.y;
        for (int k = threadIdx.x * VEC; k < d; k += kLongThreads * VEC) {
            float c[VEC], w[VEC], b[VEC];
            V v;
            v.load(xr + k);
            v.get(c);
            if (gamma) {
                v.load(gamma + k);
                v.get(w);
            }
            if (beta) {
                v.load(beta + k);
                v.get(b);
            }
#pragma unroll
            for (int q = 0; q < VEC; ++q)
                c[q] = fmaf((c[q] - st.x) * rstd, gamma ? w[q] : 1.f, beta ? b[q] : 0.f);
            V::store(y + row * d + k, c);
        }
        if (threadIdx.x == 0) {
            if (mean_out) mean_out[row] = st.x;
            if (rstd_out) rstd_out[row] = rstd;
        }
    }
}

// stats [T]: (mu, 1 / sigma) of every row, for the column sums; null: not wanted.
template <typename TT, int VEC>
__global__ void __launch_bounds__(kLongThreads)
    layernorm_vjp_long_kernel(const TT* __restrict__ g, const TT* __restrict__ x,
                              const TT* __restrict__ gamma, int T, int d, float eps, float min_rms,
                              TT* __restrict__ out, float2* __restrict__ stats) {
    using V = RowVec<TT, VEC>;
    __shared__ float sh[2][2][kLongThreads / 32];
    RowSum<2, kLongThreads / 32> sum{&sh, 0, 0};
    grid_dependency_trigger();
    const float inv_d = 1.f / static_cast<float>(d);
    for (long long row = blockIdx.x; row < T; row += gridDim.x) {
        const TT* xr = x + row * d;
        const TT* gr = g + row * d;
        const float2 st = long_stats<TT, VEC>(xr, d, eps, sum);
        const float mu = st.x, rstd = 1.f / st.y, pref = 1.f / fmaxf(st.y, min_rms);
        if (stats && threadIdx.x == 0) stats[row] = make_float2(mu, rstd);
        if (!out) continue;
        float s[2] = {0.f, 0.f};  // u, u xhat
        auto vec = [&](int k, float(&u)[VEC], float(&xh)[VEC]) {
            V v;
            v.load(xr + k);
            v.get(xh);
            v.load(gr + k);
            v.get(u);
            float w[VEC];
            if (gamma) {
                v.load(gamma + k);
                v.get(w);
            }
#pragma unroll
            for (int q = 0; q < VEC; ++q) {
                u[q] *= gamma ? w[q] : 1.f;
                xh[q] = (xh[q] - mu) * rstd;
            }
        };
        for (int k = threadIdx.x * VEC; k < d; k += kLongThreads * VEC) {
            float u[VEC], xh[VEC];
            vec(k, u, xh);
#pragma unroll
            for (int q = 0; q < VEC; ++q) {
                s[0] += u[q];
                s[1] = fmaf(u[q], xh[q], s[1]);
            }
        }
        sum(s);
        const float um = s[0] * inv_d, cm = s[1] * inv_d;
        for (int k = threadIdx.x * VEC; k < d; k += kLongThreads * VEC) {
            float u[VEC], xh[VEC];
            vec(k, u, xh);
#pragma unroll
            for (int q = 0; q < VEC; ++q) u[q] = fmaf(-xh[q], cm, u[q] - um) * pref;
            V::store(out + row * d + k, u);
        }
    }
}

// Column sums of long rows: block (column tile, row range) of 256 columns, one per thread.
constexpr int kColThreads = 256;
template <typename TT>
__global__ void __launch_bounds__(kColThreads)
    layernorm_cols_kernel(const TT* g, const TT* x, const float2* stats,
                          int T, int d, float* part) {
    grid_dependency_trigger();
    grid_dependency_wait();
    const int k = blockIdx.x * kColThreads + threadIdx.x;
    if (k >= d) return;
    const int r0 = static_cast<int>(static_cast<long long>(blockIdx.y) * T / gridDim.y);
    const int r1 = static_cast<int>(static_cast<long long>(blockIdx.y + 1) * T / gridDim.y);
    float dg = 0.f, db = 0.f;
#pragma unroll 4
    for (int r = r0; r < r1; ++r) {
        const float2 st = stats[r];
        const size_t o = static_cast<size_t>(r) * d + k;
        const float gv = static_cast<float>(g[o]);
        dg = fmaf(gv, (static_cast<float>(x[o]) - st.x) * st.y, dg);
        db += gv;
    }
    float* p = part + static_cast<size_t>(blockIdx.y) * 2 * d;
    p[k] = dg;
    p[d + k] = db;
}

// dgamma, dbeta [d] from part [n][2][d]: 32 columns per block, 16 threads to a column, each
// a contiguous range of the n; the ranges' sums in order.
constexpr int kFinCols = 32, kFinRanges = 16;
__global__ void __launch_bounds__(kFinCols* kFinRanges)
    layernorm_cols_final_kernel(const float* part, int n, int d, float* dgamma, float* dbeta) {
    __shared__ float sh[kFinRanges][kFinCols];
    grid_dependency_wait();
    const int c = threadIdx.x % kFinCols, r = threadIdx.x / kFinCols;
    const int col = static_cast<int>(blockIdx.x) * kFinCols + c;  // of the 2 d
    float a = 0.f;
    if (col < 2 * d) {
        const int i0 = r * n / kFinRanges, i1 = (r + 1) * n / kFinRanges;
#pragma unroll 8
        for (int i = i0; i < i1; ++i) a += part[static_cast<size_t>(i) * 2 * d + col];
    }
    sh[r][c] = a;
    __syncthreads();
    if (r != 0 || col >= 2 * d) return;
#pragma unroll
    for (int i = 1; i < kFinRanges; ++i) a += sh[i][c];
    if (col < d) {
        if (dgamma) dgamma[col] = a;
    } else if (dbeta) {
        dbeta[col - d] = a;
    }
}

// Vectors per thread and threads per row of the register kernels for rows of d elements in
// vectors of VEC: the fewest threads (a row's sums then cross few warps, and several rows share
// an SM), up to 512.
struct RowForm {
    int nv, th;  // 0: a long row
};
template <typename TT, int VEC>
RowForm row_form(int d) {
    constexpr int kMax = ln_ept<TT>() / VEC, kMax512 = ln_ept<TT, 512>() / VEC;
    const int n = (d + VEC - 1) / VEC;
    for (int nv = 1; nv <= kMax; nv *= 2)
        if (n <= 32 * nv) return {nv, 32};
    for (int th = 64; th <= 256; th *= 2)
        if (n <= th * kMax) return {kMax, th};
    if (n <= 512 * kMax512) return {kMax512, 512};
    return {0, 0};
}

int sms() {
    DevInfo di;
    return current_device_info(&di) ? di.sm_count : 152;
}

// Blocks of the register kernels of the backward pass, each with its share of the weight
// sums: as many as are resident on 152 SMs (ln_min_blocks).
int vjp_blocks(int T, const RowForm& f) {
    const int rows = f.th == 512 ? 1 : 256 / f.th, cap = f.th == 512 ? 152 : 304;
    const int want = T / rows + (T % rows != 0);
    return want < cap ? want : cap;
}
// Short batches: all of it on one cluster, in at most kLnClusterRounds rounds over the blocks'
// row groups.  bf16 200 x 256, 4 rounds: a call takes 7.7 us, 16.2 on the two kernels with a
// fresh workspace (4.8 and 3.7 us on the GPU, in a graph); at 8 rounds (512 x 256) 8.4 and
// 16.5, but 6.8 and 4.1 on the GPU.
constexpr int kLnClusterRounds = 4;
bool one_cluster(int T, const RowForm& f) {
    return f.nv != 0 && f.th != 512 && T <= kLnClusterRounds * kLnCluster * (256 / f.th);
}
constexpr int kLongRanges = 64;
int long_ranges(int T) { return T < kLongRanges ? T : kLongRanges; }

// Calls f with (vectors per thread, threads per row) as compile-time constants.
template <int N>
struct Int {
    static constexpr int value = N;
};
template <typename TT, int VEC, class F>
cudaError_t with_form(const RowForm& f, F&& fn) {
    constexpr int kMax = ln_ept<TT>() / VEC, kMax512 = ln_ept<TT, 512>() / VEC;
    switch (f.th) {
        case 64: return fn(Int<kMax>{}, Int<64>{});
        case 128: return fn(Int<kMax>{}, Int<128>{});
        case 256: return fn(Int<kMax>{}, Int<256>{});
        case 512: return fn(Int<kMax512>{}, Int<512>{});
        default: break;
    }
    if constexpr (kMax >= 16) {
        if (f.nv == 16) return fn(Int<16>{}, Int<32>{});
    }
    if constexpr (kMax >= 8) {
        if (f.nv == 8) return fn(Int<8>{}, Int<32>{});
    }
    if constexpr (kMax >= 4) {
        if (f.nv == 4) return fn(Int<4>{}, Int<32>{});
    }
    if constexpr (kMax >= 2) {
        if (f.nv == 2) return fn(Int<2>{}, Int<32>{});
    }
    return fn(Int<1>{}, Int<32>{});
}

template <typename TT, int VEC>
cudaError_t run_fwd(const void* x, const void* gamma, const void* beta, int T, int d, float eps,
                    void* y, float* mean_out, float* rstd_out, cudaStream_t st) {
    const auto* xx = static_cast<const TT*>(x);
    const auto* gg = static_cast<const TT*>(gamma);
    const auto* bb = static_cast<const TT*>(beta);
    auto* yy = static_cast<TT*>(y);
    const RowForm f = row_form<TT, VEC>(d);
    if (f.nv == 0) {
        const int grid = T < 4 * sms() ? T : 4 * sms();
        layernorm_fwd_long_kernel<TT, VEC>
            <<<grid, kLongThreads, 0, st>>>(xx, gg, bb, T, d, eps, yy, mean_out, rstd_out),
            note_launch();
        return cudaGetLastError();
    }
    return with_form<TT, VEC>(f, [&](auto nv, auto th) {
        constexpr int NV = decltype(nv)::value, TH = decltype(th)::value;
        const int blocks = T / ln_rows<TH>() + (T % ln_rows<TH>() != 0);
        const int cap = sms() * ln_min_blocks<TH, false>();
        layernorm_fwd_kernel<TT, VEC, NV, TH>
            <<<blocks < cap ? blocks : cap, ln_threads<TH>(), 0, st>>>(xx, gg, bb, T, d, eps, yy,
                                                                      mean_out, rstd_out),
            note_launch();
        return cudaGetLastError();
    });
}

template <typename TT, int VEC>
cudaError_t run_vjp(const void* g, const void* x, const void* gamma, int T, int d, float eps,
                    float min_rms, void* out, float* dgamma, float* dbeta, float* ws,
                    cudaStream_t st) {
    const auto* gg = static_cast<const TT*>(g);
    const auto* xx = static_cast<const TT*>(x);
    const auto* ww = static_cast<const TT*>(gamma);
    auto* oo = static_cast<TT*>(out);
    const bool sums = dgamma || dbeta;
    const RowForm f = row_form<TT, VEC>(d);
    int parts = 0;
    cudaError_t e;
    if (f.nv == 0) {
        float2* stats = sums ? reinterpret_cast<float2*>(ws) : nullptr;
        const int grid = T < 4 * sms() ? T : 4 * sms();
        layernorm_vjp_long_kernel<TT, VEC>
            <<<grid, kLongThreads, 0, st>>>(gg, xx, ww, T, d, eps, min_rms, oo, stats),
            note_launch();
        e = cudaGetLastError();
        if (e != cudaSuccess || !sums) return e;
        ws += 2 * static_cast<size_t>(T);
        parts = long_ranges(T);
        e = launch_chained(layernorm_cols_kernel<TT>,
                           dim3((d + kColThreads - 1) / kColThreads, parts), kColThreads, 0, st, gg,
                           xx, static_cast<const float2*>(stats), T, d, ws);
    } else if (sums && one_cluster(T, f)) {
        return with_form<TT, VEC>(f, [&](auto nv, auto th) {
            constexpr int NV = decltype(nv)::value, TH = decltype(th)::value;
            if constexpr (TH != 512) {
                cudaLaunchConfig_t cfg = {};
                cfg.gridDim = dim3(kLnCluster, 1, 1);
                cfg.blockDim = dim3(ln_threads<TH>(), 1, 1);
                cfg.stream = st;
                cudaLaunchAttribute at[1];
                at[0].id = cudaLaunchAttributeClusterDimension;
                at[0].val.clusterDim.x = kLnCluster;
                at[0].val.clusterDim.y = at[0].val.clusterDim.z = 1;
                cfg.attrs = at;
                cfg.numAttrs = 1;
                note_launch();
                return cudaLaunchKernelEx(&cfg, layernorm_vjp_kernel<TT, VEC, NV, TH, kClusterSums>,
                                          gg, xx, ww, T, d, eps, min_rms, oo,
                                          static_cast<float*>(nullptr), dgamma, dbeta);
            } else {
                return cudaErrorInvalidValue;  // (one_cluster)
            }
        });
    } else {
        parts = vjp_blocks(T, f);
        e = with_form<TT, VEC>(f, [&](auto nv, auto th) {
            constexpr int NV = decltype(nv)::value, TH = decltype(th)::value;
            if (sums)
                layernorm_vjp_kernel<TT, VEC, NV, TH, kPartSums><<<parts, ln_threads<TH>(), 0, st>>>(
                    gg, xx, ww, T, d, eps, min_rms, oo, ws, nullptr, nullptr),
                    note_launch();
            else
                layernorm_vjp_kernel<TT, VEC, NV, TH, kNoSums><<<parts, ln_threads<TH>(), 0, st>>>(
                    gg, xx, ww, T, d, eps, min_rms, oo, nullptr, nullptr, nullptr),
                    note_launch();
            return cudaGetLastError();
        });
    }
    if (e != cudaSuccess || !sums) return e;
    return launch_chained(layernorm_cols_final_kernel, dim3((2 * d + kFinCols - 1) / kFinCols),
                          kFinCols * kFinRanges, 0, st, static_cast<const float*>(ws), parts, d,
                          dgamma, dbeta);
}

}  // namespace

size_t layernorm_vjp_floats(int dtype, int T, int d) {
    const RowForm f = dtype == 1   ? row_form<__nv_bfloat16, 8>(d)
                      : d % 4 == 0 ? row_form<float, 4>(d)
                                   : row_form<float, 1>(d);
    if (one_cluster(T, f)) return 0;
    const size_t stats = f.nv == 0 ? 2 * static_cast<size_t>(T) : 0;
    const size_t parts = f.nv == 0 ? long_ranges(T) : vjp_blocks(T, f);
    return stats + parts * 2 * static_cast<size_t>(d);
}

cudaError_t launch_layernorm_fwd(int dtype, const void* x, const void* gamma, const void* beta,
                                 int T, int d, float eps, void* y, float* mean_out,
                                 float* rstd_out, cudaStream_t st) {
    if (T <= 0) return cudaSuccess;
    if (dtype == 1)
        return run_fwd<__nv_bfloat16, 8>(x, gamma, beta, T, d, eps, y, mean_out, rstd_out, st);
    if (d % 4 == 0) return run_fwd<float, 4>(x, gamma, beta, T, d, eps, y, mean_out, rstd_out, st);
    return run_fwd<float, 1>(x, gamma, beta, T, d, eps, y, mean_out, rstd_out, st);
}

cudaError_t launch_layernorm_vjp(int dtype, const void* g, const void* x, const void* gamma, int T,
                                 int d, float eps, float min_rms, void* out, float* dgamma,
                                 float* dbeta, float* ws, cudaStream_t st) {
    if (T <= 0) return cudaSuccess;
    if (dtype == 1)
        return run_vjp<__nv_bfloat16, 8>(g, x, gamma, T, d, eps, min_rms, out, dgamma, dbeta, ws, st);
    if (d % 4 == 0)
        return run_vjp<float, 4>(g, x, gamma, T, d, eps, min_rms, out, dgamma, dbeta, ws, st);
    return run_vjp<float, 1>(g, x, gamma, T, d, eps, min_rms, out, dgamma, dbeta, ws, st);
}

}  // namespace fpo
