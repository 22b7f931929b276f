// layernorm.cu -- LayerNorm over the rows of x [T, d] and its backward pass, for model
// families whose blocks normalise with the mean removed.
//
//   forward   mu = mean_j x_j, sigma = sqrt(mean_j (x_j - mu)^2 + eps)
//             y = gamma (.) (x - mu) / sigma + beta
//   backward  xhat = (x - mu) / sigma, u = gamma (.) g
//             g_out = (u - mean(u) - xhat mean(u (.) xhat)) / max(sigma, min_rms)
//             dgamma = sum_t g_t (.) xhat_t,  dbeta = sum_t g_t
//
// Rows of up to 8192 elements stay in a block's registers and are read once: the variance is the sum of squares around the row's own mean (a difference of two large
// sums would lose it), and the backward pass forms mu and sigma again from the row that it
// has to read anyway, so no statistics are saved between the passes.  A row's next vectors
// are loaded before the reductions of the one at hand.  Each thread keeps the same columns
// for every row of its block, so the weight sums stay in its registers until the last row;
// the blocks' sums are then added in block order by a second kernel (no atomics: repeat calls
// give identical bits).  Longer rows go through the row in several passes, and their weight
// sums through a kernel of their own.
//
// Bound: HBM.
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <math.h>

#include "internal.h"

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
// butterfly per warp, then the warps' sums in warp order.  `buf` alternates between two
// areas from call to call, so one barrier a call is enough.
template <int N, int W>
struct RowSum {
    float (*sh)[2][N][W];  // shared (W > 1 only)
    int at;
    __device__ __forceinline__ void operator()(float (&v)[N]) {
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) {
#pragma unroll
            for (int k = 0; k < N; ++k) v[k] += __shfl_xor_sync(0xffffffffu, v[k], o);
        }
        if constexpr (W > 1) {
            const int w = threadIdx.x >> 5;
            if ((threadIdx.x & 31) == 0) {
#pragma unroll
                for (int k = 0; k < N; ++k) (*sh)[at][k][w] = v[k];
            }
            __syncthreads();
#pragma unroll
            for (int k = 0; k < N; ++k) {
                v[k] = 0.f;
#pragma unroll
                for (int i = 0; i < W; ++i) v[k] += (*sh)[at][k][i];
            }
            at ^= 1;
        }
    }
};

// TH threads to a row (a warp: 8 rows per block), NV vectors of VEC elements per thread:
// vector v of thread t holds elements (v TH + t) VEC ...
template <int TH>
constexpr int ln_threads() {
    return TH == 32 ? 256 : TH;
}
template <int TH>
constexpr int ln_rows() {
    return ln_threads<TH>() / TH;
}

template <typename TT, int VEC, int NV, int TH>
__global__ void __launch_bounds__(ln_threads<TH>())
    layernorm_fwd_kernel(const TT* __restrict__ x, const TT* __restrict__ gamma,
                         const TT* __restrict__ beta, int T, int d, float eps,
                         TT* __restrict__ y, float* __restrict__ mean_out,
                         float* __restrict__ rstd_out) {
    using V = RowVec<TT, VEC>;
    constexpr int kW = TH / 32;
    __shared__ float sh[2][1][kW];
    RowSum<1, kW> row_sum{&sh, 0};
    const int t = threadIdx.x % TH;
    const float inv_d = 1.f / static_cast<float>(d);
    V nx[NV];
    auto load = [&](long long row) {
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            const int k = (v * TH + t) * VEC;
            if (k < d)
                nx[v].load(x + row * d + k);
            else
                nx[v].zero();
        }
    };
    const long long step = gridDim.x * ln_rows<TH>();
    long long row = blockIdx.x * ln_rows<TH>() + threadIdx.x / TH;
    if (row < T) load(row);
    for (; row < T; row += step) {
        float c[NV][VEC];
        float s[1] = {0.f};
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            nx[v].get(c[v]);
#pragma unroll
            for (int q = 0; q < VEC; ++q) s[0] += c[v][q];
        }
        if (row + step < T) load(row + step);
        row_sum(s);
        const float mu = __fmul_rn(s[0], inv_d);
        s[0] = 0.f;
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            const bool in = (v * TH + t) * VEC < d;
#pragma unroll
            for (int q = 0; q < VEC; ++q) {
                c[v][q] = in ? c[v][q] - mu : 0.f;
                s[0] = fmaf(c[v][q], c[v][q], s[0]);
            }
        }
        row_sum(s);
        const float rstd = 1.f / sqrtf(fmaf(s[0], inv_d, eps));
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            const int k = (v * TH + t) * VEC;
            if (k >= d) continue;
            float w[VEC], b[VEC], o[VEC];
            V u;
            if (gamma) {
                u.load(gamma + k);
                u.get(w);
            }
            if (beta) {
                u.load(beta + k);
                u.get(b);
            }
#pragma unroll
            for (int q = 0; q < VEC; ++q)
                o[q] = fmaf(c[v][q] * rstd, gamma ? w[q] : 1.f, beta ? b[q] : 0.f);
            V::store(y + row * d + k, o);
        }
        if (t == 0) {
            if (mean_out) mean_out[row] = mu;
            if (rstd_out) rstd_out[row] = rstd;
        }
    }
}

// part (kW only): [grid][2][d] sums of g xhat and of g over the block's rows.
template <typename TT, int VEC, int NV, int TH, bool kSums>
__global__ void __launch_bounds__(ln_threads<TH>())
    layernorm_vjp_kernel(const TT* __restrict__ g, const TT* __restrict__ x,
                         const TT* __restrict__ gamma, int T, int d, float eps, float min_rms,
                         TT* __restrict__ out, float* __restrict__ part) {
    using V = RowVec<TT, VEC>;
    constexpr int kW = TH / 32;
    __shared__ float sh1[2][2][kW], sh2[2][2][kW];
    RowSum<2, kW> sum1{&sh1, 0}, sum2{&sh2, 0};
    grid_dependency_trigger();
    const int t = threadIdx.x % TH;
    const float inv_d = 1.f / static_cast<float>(d);
    V nx[NV], ng[NV], w[NV];
#pragma unroll
    for (int v = 0; v < NV; ++v) {
        w[v].zero();
        const int k = (v * TH + t) * VEC;
        if (gamma && k < d) w[v].load(gamma + k);
    }
    auto load = [&](long long row) {
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            const int k = (v * TH + t) * VEC;
            if (k < d) {
                nx[v].load(x + row * d + k);
                ng[v].load(g + row * d + k);
            } else {
                nx[v].zero();
                ng[v].zero();
            }
        }
    };
    float dg[kSums ? NV : 1][VEC], db[kSums ? NV : 1][VEC];
#pragma unroll
    for (int v = 0; v < (kSums ? NV : 1); ++v) {
#pragma unroll
        for (int q = 0; q < VEC; ++q) dg[v][q] = db[v][q] = 0.f;
    }
    const long long step = gridDim.x * ln_rows<TH>();
    long long row = blockIdx.x * ln_rows<TH>() + threadIdx.x / TH;
    if (row < T) load(row);
    for (; row < T; row += step) {
        float c[NV][VEC], gv[NV][VEC];
        float s[2] = {0.f, 0.f};  // x, then u
        auto weight = [&](int v, int q) {
            float wv[VEC];
            w[v].get(wv);
            return gamma ? wv[q] : 1.f;
        };
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            nx[v].get(c[v]);
            ng[v].get(gv[v]);
#pragma unroll
            for (int q = 0; q < VEC; ++q) {
                s[0] += c[v][q];
                s[1] = fmaf(gv[v][q], weight(v, q), s[1]);
            }
        }
        if (row + step < T) load(row + step);
        sum1(s);
        // (explicit roundings and FMAs from here: the same bits with and without the sums)
        const float mu = __fmul_rn(s[0], inv_d), um = __fmul_rn(s[1], inv_d);
        s[0] = s[1] = 0.f;  // (x - mu)^2, then u (x - mu)
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            const bool in = (v * TH + t) * VEC < d;
#pragma unroll
            for (int q = 0; q < VEC; ++q) {
                c[v][q] = in ? c[v][q] - mu : 0.f;
                s[0] = fmaf(c[v][q], c[v][q], s[0]);
                s[1] = fmaf(__fmul_rn(gv[v][q], weight(v, q)), c[v][q], s[1]);
            }
        }
        sum2(s);
        const float sigma = sqrtf(fmaf(s[0], inv_d, eps));
        const float rstd = 1.f / sigma;
        const float cm = __fmul_rn(__fmul_rn(s[1], inv_d), rstd);  // mean(u xhat)
        const float pref = 1.f / fmaxf(sigma, min_rms);
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            const int k = (v * TH + t) * VEC;
            float o[VEC];
#pragma unroll
            for (int q = 0; q < VEC; ++q) {
                const float xh = __fmul_rn(c[v][q], rstd);
                o[q] = fmaf(-xh, cm, fmaf(gv[v][q], weight(v, q), -um)) * pref;
                if constexpr (kSums) {
                    dg[v][q] = fmaf(gv[v][q], xh, dg[v][q]);
                    db[v][q] += gv[v][q];
                }
            }
            if (out && k < d) V::store(out + row * d + k, o);
        }
    }
    if constexpr (kSums) {
        float* p = part + static_cast<size_t>(blockIdx.x) * 2 * d;
        if constexpr (ln_rows<TH>() > 1) {
            // the block's 8 warps hold the same columns: their sums in warp order
            constexpr int kCols = NV * TH * VEC;
            __shared__ float acc[ln_rows<TH>()][kCols];
#pragma unroll
            for (int which = 0; which < 2; ++which) {
                __syncthreads();
#pragma unroll
                for (int v = 0; v < NV; ++v) {
#pragma unroll
                    for (int q = 0; q < VEC; ++q)
                        acc[threadIdx.x / TH][(v * TH + t) * VEC + q] = which ? db[v][q] : dg[v][q];
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
#pragma unroll
            for (int v = 0; v < NV; ++v) {
#pragma unroll
                for (int q = 0; q < VEC; ++q) {
                    const int k = (v * TH + t) * VEC + q;
                    if (k < d) {
                        p[k] = dg[v][q];
                        p[d + k] = db[v][q];
                    }
                }
            }
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
    RowSum<2, kLongThreads / 32> sum{&sh, 0};
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
    RowSum<2, kLongThreads / 32> sum{&sh, 0};
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

// dgamma, dbeta [d] from part [n][2][d]: 32 columns per block, 8 threads to a column, each
// a contiguous range of the n; the ranges' sums in order.
constexpr int kFinCols = 32, kFinRanges = 8;
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
// vectors of vec; up to 16 elements per thread (with 32 the backward pass's sums spill).
struct RowForm {
    int nv, th;  // 0: a long row
};
RowForm row_form(int d, int vec) {
    const int n = (d + vec - 1) / vec;
    if (n <= 32) return {1, 32};
    if (n <= 64) return {2, 32};
    if (n <= 128) return {1, 128};
    if (n <= 256) return {1, 256};
    for (int nv = 1; nv * vec <= 16; nv *= 2)
        if (n <= 512 * nv) return {nv, 512};
    return {0, 0};
}

int sms() {
    DevInfo di;
    return current_device_info(&di) ? di.sm_count : 152;
}

// Blocks of the register kernels of the backward pass, each with its share of the weight
// sums: enough for two of 512 threads (more of the smaller ones) on each of 152 SMs.
int vjp_blocks(int T, const RowForm& f) {
    const int rows = f.th == 32 ? 8 : 1, cap = f.th == 512 ? 304 : 608;
    const int want = T / rows + (T % rows != 0);
    return want < cap ? want : cap;
}
constexpr int kLongRanges = 64;
int long_ranges(int T) { return T < kLongRanges ? T : kLongRanges; }

int vec_of(int dtype, int d) { return dtype == 1 ? 8 : d % 4 == 0 ? 4 : 1; }

// Calls f with (vectors per thread, threads per row) as compile-time constants.
template <int N>
struct Int {
    static constexpr int value = N;
};
template <int VEC, class F>
cudaError_t with_form(const RowForm& f, F&& fn) {
    if (f.th == 32) return f.nv == 1 ? fn(Int<1>{}, Int<32>{}) : fn(Int<2>{}, Int<32>{});
    if (f.th == 128) return fn(Int<1>{}, Int<128>{});
    if (f.th == 256) return fn(Int<1>{}, Int<256>{});
    if (f.nv == 1) return fn(Int<1>{}, Int<512>{});
    if constexpr (VEC <= 4) {
        if (f.nv == 4) return fn(Int<4>{}, Int<512>{});
    }
    if constexpr (VEC == 1) {
        if (f.nv == 8) return fn(Int<8>{}, Int<512>{});
        if (f.nv == 16) return fn(Int<16>{}, Int<512>{});
    }
    return fn(Int<2>{}, Int<512>{});
}

template <typename TT, int VEC>
cudaError_t run_fwd(const void* x, const void* gamma, const void* beta, int T, int d, float eps,
                    void* y, float* mean_out, float* rstd_out, cudaStream_t st) {
    const auto* xx = static_cast<const TT*>(x);
    const auto* gg = static_cast<const TT*>(gamma);
    const auto* bb = static_cast<const TT*>(beta);
    auto* yy = static_cast<TT*>(y);
    const RowForm f = row_form(d, VEC);
    if (f.nv == 0) {
        const int grid = T < 4 * sms() ? T : 4 * sms();
        layernorm_fwd_long_kernel<TT, VEC>
            <<<grid, kLongThreads, 0, st>>>(xx, gg, bb, T, d, eps, yy, mean_out, rstd_out),
            note_launch();
        return cudaGetLastError();
    }
    return with_form<VEC>(f, [&](auto nv, auto th) {
        constexpr int NV = decltype(nv)::value, TH = decltype(th)::value;
        const int blocks = T / ln_rows<TH>() + (T % ln_rows<TH>() != 0);
        const int cap = sms() * (2048 / ln_threads<TH>());
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
    const RowForm f = row_form(d, VEC);
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
    } else {
        parts = vjp_blocks(T, f);
        e = with_form<VEC>(f, [&](auto nv, auto th) {
            constexpr int NV = decltype(nv)::value, TH = decltype(th)::value;
            if (sums)
                layernorm_vjp_kernel<TT, VEC, NV, TH, true><<<parts, ln_threads<TH>(), 0, st>>>(
                    gg, xx, ww, T, d, eps, min_rms, oo, ws),
                    note_launch();
            else
                layernorm_vjp_kernel<TT, VEC, NV, TH, false><<<parts, ln_threads<TH>(), 0, st>>>(
                    gg, xx, ww, T, d, eps, min_rms, oo, nullptr),
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
    const int vec = vec_of(dtype, d);
    const RowForm f = row_form(d, vec);
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
