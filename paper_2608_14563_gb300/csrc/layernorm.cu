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
// atomics: repeat calls give identical bits).  Large batches of long rows go through a ring in
// shared memory instead, with the roles on warps of their own.  Rows of more than 8192 elements
// are read in several passes, and their weight sums by a kernel of their own.
//
// Bound: HBM.  bf16 16384 x 4096, call after call: forward 50 us, 5.4 TB/s; backward with both
// weight gradients 76 us, 5.3 TB/s.  Small calls are bound by the host (a call is 7 to 8 us of it,
// 2 to 5 on the GPU).
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

// An untiled bulk copy of `bytes` (a multiple of 16, both addresses on 16 bytes) to shared memory,
// counted on `bar`.
__device__ __forceinline__ void bulk_load(uint32_t dst, const void* src, uint32_t bytes,
                                          uint32_t bar) {
    asm volatile(
        "cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::
            "r"(dst),
        "l"(reinterpret_cast<uint64_t>(src)), "r"(bytes), "r"(bar)
        : "memory");
}

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

// ------------------------------------------------------------------ many rows
// The backward pass of large batches of long rows.  A block's rows pass through a ring in
// shared memory: a loader warp fills the slots with bulk copies, SW warps form the statistics
// of a row each, and CW warps, whose threads keep the same NV vectors of columns throughout,
// apply them in row order.  A row costs 25 shuffles and no barrier of the block; with a row's
// sums over 256 threads (layernorm_vjp_kernel) 256 shuffles and two barriers of the block were
// most of its time.  bf16 16384 x 4096: 76 us with the last sums (floor 59), 93 there.
//
// The statistics take one pass, with the mean s of the row's first 32 vectors as the origin:
//   var = mean((x - s)^2) - mean(x - s)^2,  mean(u (x - mu)) = mean(u (x - s)) - mean(x - s) mean(u)
// The differences lose digits where s is far from mu: with n elements in s, (s - mu)^2 can be
// (d / n) sigma^2.  A row with (s - mu)^2 > sigma^2 takes a second pass around its mean, so at most a
// factor of 4 of the 24 bits is lost.  (In a random row (s - mu)^2 is about sigma^2 / n.  Two passes
// for every row, bf16 8192 x 8192: 101 us, 90 with this rule.)
//
// Every wait is bounded.  One that runs out ends the block, whose warps leave NaN in the rows (of
// their columns) that they did not reach, and in their weight sums.
constexpr int kLnMaxSlots = 16;
constexpr int kLnStreamSmem = 220 * 1024;  // of dynamic shared memory: weights and slots

template <int CW, int SW>
struct LnStream {
    static constexpr int kThreads = 32 * (CW + SW + 1);
};

__device__ __forceinline__ bool ln_wait(uint32_t bar, uint32_t parity, volatile int* lost,
                                        uint64_t limit_ns) {
    if (mbar_try_wait(bar, parity)) return true;
    const uint64_t t0 = global_timer_ns();
    while (!mbar_try_wait(bar, parity)) {
        if (*lost) return false;
        if (global_timer_ns() - t0 > limit_ns) {
            *lost = 1;
            return false;
        }
    }
    return true;
}

// Mean of a row's first 32 vectors (inv_n: 1 / their elements), in every lane of the warp.
template <typename TT, int VEC>
__device__ __forceinline__ float ln_origin(const TT* xs, int lane, int n, float inv_n) {
    float a = 0.f;
    if (lane < n) {
        float v[VEC];
        RowVec<TT, VEC> r;
        r.load(xs + lane * VEC);
        r.get(v);
#pragma unroll
        for (int q = 0; q < VEC; ++q) a += v[q];
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) a += __shfl_xor_sync(0xffffffffu, a, o);
    return a * inv_n;
}

// Whether a row's statistics around an origin that is `off` from its mean need a second pass around
// the mean (not for a NaN).
__device__ __forceinline__ bool ln_far(float off, float square) { return 2.f * off * off > square; }

// mean((x - s)^2) - mean(x - s)^2, not below zero (a NaN stays one).
__device__ __forceinline__ float ln_variance(float off, float square) {
    const float v = fmaf(-off, off, square);
    return v < 0.f ? 0.f : v;
}

// The loader's end: the last min(slots, filled) copies are waited for, whatever the wait limit, so
// that the block leaves none in flight.
__device__ __forceinline__ void ln_drain(uint64_t* full, int slots, int filled) {
    for (int j = filled > slots ? filled - slots : 0; j < filled; ++j)
        mbar_wait_drain(smem_u32(&full[j % slots]), (j / slots) & 1, 2000000000ull);
}

// Rows of block b of `blocks`: b, b + blocks, ... below T.
__device__ __forceinline__ int ln_block_rows(int T) {
    return static_cast<int>((T - static_cast<long long>(blockIdx.x) + gridDim.x - 1) / gridDim.x);
}
__device__ __forceinline__ long long ln_block_row(int i) {
    return blockIdx.x + static_cast<long long>(i) * gridDim.x;
}

// The forward pass: every warp takes whole rows from the ring, so a row costs it 15 shuffles and
// no barrier of the block.
constexpr int kLnFwdWarps = 16;
template <typename TT, int VEC>
__global__ void __launch_bounds__(32 * (kLnFwdWarps + 1), 1)
    layernorm_fwd_stream_kernel(const TT* __restrict__ x, const TT* __restrict__ gamma,
                                const TT* __restrict__ beta, int T, int d, float eps,
                                TT* __restrict__ y, float* __restrict__ mean_out,
                                float* __restrict__ rstd_out, int slots, uint64_t limit_ns) {
    using V = RowVec<TT, VEC>;
    extern __shared__ __align__(16) char ln_smem[];
    __shared__ uint64_t full[kLnMaxSlots], empty[kLnMaxSlots];
    __shared__ int lost_word;
    volatile int* lost = &lost_word;
    TT* const w_sm = reinterpret_cast<TT*>(ln_smem);
    TT* const b_sm = w_sm + d;
    TT* const ring = b_sm + d;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    if (threadIdx.x == 0) {
        for (int i = 0; i < slots; ++i) {
            mbar_init(smem_u32(&full[i]), 1);
            mbar_init(smem_u32(&empty[i]), 1);
        }
        lost_word = 0;
        fence_mbar_init();
    }
    for (int k = threadIdx.x * VEC; k < d; k += 32 * (kLnFwdWarps + 1) * VEC) {
        V v;
        if (gamma) {
            v.load(gamma + k);
            *reinterpret_cast<V*>(w_sm + k) = v;
        }
        if (beta) {
            v.load(beta + k);
            *reinterpret_cast<V*>(b_sm + k) = v;
        }
    }
    __syncthreads();
    const int rows = ln_block_rows(T);
    if (warp == kLnFwdWarps) {
        if (lane == 0) {
            const uint32_t bytes = static_cast<uint32_t>(d) * sizeof(TT);
            int s = 0, i = 0;
            uint32_t phase = 0;
            for (; i < rows; ++i) {
                if (i >= slots && !ln_wait(smem_u32(&empty[s]), phase ^ 1u, lost, limit_ns)) break;
                mbar_arrive_expect_tx(smem_u32(&full[s]), bytes);
                bulk_load(smem_u32(ring + static_cast<size_t>(s) * d), x + ln_block_row(i) * d, bytes,
                          smem_u32(&full[s]));
                if (++s == slots) { s = 0; phase ^= 1u; }
            }
            ln_drain(full, slots, i);
        }
        return;
    }
    const int n = d / VEC;
    const float inv_d = 1.f / static_cast<float>(d);
    const float inv_n = 1.f / static_cast<float>(VEC * (n < 32 ? n : 32));
    // (a slot is always the same warp's, so its waits cannot mistake a phase)
    const int warps = slots < kLnFwdWarps ? slots : kLnFwdWarps;
    int i = warp < warps ? warp : rows;
    for (; i < rows; i += warps) {
        const int s = i % slots;
        if (!__all_sync(0xffffffffu, ln_wait(smem_u32(&full[s]), (i / slots) & 1, lost, limit_ns)))
            break;
        const TT* xs = ring + static_cast<size_t>(s) * d;
        float origin = ln_origin<TT, VEC>(xs, lane, n, inv_n);
        float off, square;  // mean(x - origin), mean((x - origin)^2)
        for (int pass = 0;; ++pass) {
            const float2 shift = both(-origin);
            float2 a0 = both(0.f), a1 = a0;
            for (int k = lane * VEC; k < d; k += 32 * VEC) {
                float v[VEC];
                V r;
                r.load(xs + k);
                r.get(v);
#pragma unroll
                for (int q = 0; q < VEC; q += 2) {
                    const float2 c = __fadd2_rn(make_float2(v[q], v[q + 1]), shift);
                    a0 = __fadd2_rn(a0, c);
                    a1 = __ffma2_rn(c, c, a1);
                }
            }
            float v2[2] = {a0.x + a0.y, a1.x + a1.y};
#pragma unroll
            for (int o = 16; o > 0; o >>= 1) {
                v2[0] += __shfl_xor_sync(0xffffffffu, v2[0], o);
                v2[1] += __shfl_xor_sync(0xffffffffu, v2[1], o);
            }
            off = v2[0] * inv_d;
            square = v2[1] * inv_d;
            if (pass != 0 || !__any_sync(0xffffffffu, ln_far(off, square))) break;
            origin += off;
        }
        const float mu = origin + off;
        const float rstd = 1.f / sqrtf(ln_variance(off, square) + eps);
        const long long row = ln_block_row(i);
        TT* yr = y + row * d;
        const float2 m2 = both(-mu), r2 = both(rstd);
        for (int k = lane * VEC; k < d; k += 32 * VEC) {
            float v[VEC], wv[VEC], bv[VEC];
            V r;
            r.load(xs + k);
            r.get(v);
            if (gamma) {
                r.load(w_sm + k);
                r.get(wv);
            }
            if (beta) {
                r.load(b_sm + k);
                r.get(bv);
            }
#pragma unroll
            for (int q = 0; q < VEC; q += 2) {
                float2 c = __fmul2_rn(__fadd2_rn(make_float2(v[q], v[q + 1]), m2), r2);
                const float2 w2 = gamma ? make_float2(wv[q], wv[q + 1]) : both(1.f);
                if (beta)
                    c = __ffma2_rn(c, w2, make_float2(bv[q], bv[q + 1]));
                else
                    c = __fmul2_rn(c, w2);
                v[q] = c.x;
                v[q + 1] = c.y;
            }
            V::store(yr + k, v);
        }
        __syncwarp();
        if (lane == 0) {
            mbar_arrive(smem_u32(&empty[s]));
            if (mean_out) mean_out[row] = mu;
            if (rstd_out) rstd_out[row] = rstd;
        }
    }
    for (; i < rows && warp < warps; i += warps) {  // given up
        const float nan = __int_as_float(0x7fffffff);
        float v[VEC];
#pragma unroll
        for (int q = 0; q < VEC; ++q) v[q] = nan;
        const long long row = ln_block_row(i);
        for (int k = lane * VEC; k < d; k += 32 * VEC) V::store(y + row * d + k, v);
        if (lane == 0) {
            if (mean_out) mean_out[row] = nan;
            if (rstd_out) rstd_out[row] = nan;
        }
    }
}

template <typename TT, int VEC, int NV, int CW, int SW, bool kSums>
__global__ void __launch_bounds__(LnStream<CW, SW>::kThreads, 1)
    layernorm_vjp_stream_kernel(const TT* __restrict__ g, const TT* __restrict__ x,
                                const TT* __restrict__ gamma, int T, int d, float eps,
                                float min_rms, TT* __restrict__ out, float* __restrict__ part,
                                int slots, uint64_t limit_ns) {
    using P = RowPart<TT, VEC, NV, 32 * CW>;
    using V = RowVec<TT, VEC>;
    constexpr int kPairs = P::kPairs;
    extern __shared__ __align__(16) char ln_smem[];
    __shared__ uint64_t full[kLnMaxSlots], ready[kLnMaxSlots], empty[kLnMaxSlots];
    __shared__ float stat[kLnMaxSlots][5];  // mu, 1 / sigma, mean u, mean(u xhat), prefactor
    __shared__ int lost_word;
    volatile int* lost = &lost_word;
    grid_dependency_trigger();
    TT* const w_sm = reinterpret_cast<TT*>(ln_smem);
    TT* const ring = w_sm + d;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    if (threadIdx.x == 0) {
        for (int i = 0; i < slots; ++i) {
            mbar_init(smem_u32(&full[i]), 1);
            mbar_init(smem_u32(&ready[i]), 1);
            mbar_init(smem_u32(&empty[i]), CW);
        }
        lost_word = 0;
        fence_mbar_init();
    }
    if (gamma)
        for (int k = threadIdx.x * VEC; k < d; k += LnStream<CW, SW>::kThreads * VEC) {
            V v;
            v.load(gamma + k);
            *reinterpret_cast<V*>(w_sm + k) = v;
        }
    __syncthreads();
    const int rows = ln_block_rows(T);
    auto slot_x = [&](int s) { return ring + static_cast<size_t>(2 * s) * d; };

    if (warp == CW + SW) {
        // ----------------------------------------------------------------- loader
        if (lane == 0) {
            const uint32_t bytes = static_cast<uint32_t>(d) * sizeof(TT);
            int s = 0, i = 0;
            uint32_t phase = 0;
            for (; i < rows; ++i) {
                if (i >= slots && !ln_wait(smem_u32(&empty[s]), phase ^ 1u, lost, limit_ns)) break;
                const uint32_t bar = smem_u32(&full[s]);
                mbar_arrive_expect_tx(bar, 2 * bytes);
                bulk_load(smem_u32(slot_x(s)), x + ln_block_row(i) * d, bytes, bar);
                bulk_load(smem_u32(slot_x(s) + d), g + ln_block_row(i) * d, bytes, bar);
                if (++s == slots) { s = 0; phase ^= 1u; }
            }
            ln_drain(full, slots, i);
        }
        __syncwarp();
    } else if (warp >= CW) {
        // ----------------------------------------------------------------- statistics
        const int n = d / VEC;  // vectors of a row
        const float inv_d = 1.f / static_cast<float>(d);
        const float inv_n = 1.f / static_cast<float>(VEC * (n < 32 ? n : 32));
        const int stride = SW < slots ? SW : slots;
        for (int i = warp - CW < stride ? warp - CW : rows; i < rows; i += stride) {
            const int s = i % slots, p = i / slots;
            // A wait tells a phase from the one before it only: the slot's last row has to be
            // gone first.  (That wait is at most one phase ahead in turn, the columns being in
            // row order and stride <= slots.)
            const bool in_time =
                (p == 0 || ln_wait(smem_u32(&empty[s]), (p - 1) & 1, lost, limit_ns)) &&
                ln_wait(smem_u32(&full[s]), p & 1, lost, limit_ns);
            if (!__all_sync(0xffffffffu, in_time)) break;
            const TT *xs = slot_x(s), *gs = xs + d;
            float origin = ln_origin<TT, VEC>(xs, lane, n, inv_n);
            float v[4];
            for (int pass = 0;; ++pass) {
                const float2 shift = both(-origin);
                float2 a0 = both(0.f), a1 = a0, a2 = a0, a3 = a0;
                for (int k = lane * VEC; k < d; k += 32 * VEC) {
                    float xv[VEC], gv[VEC], wv[VEC];
                    V r;
                    r.load(xs + k);
                    r.get(xv);
                    r.load(gs + k);
                    r.get(gv);
                    if (gamma) {
                        r.load(w_sm + k);
                        r.get(wv);
                    }
#pragma unroll
                    for (int q = 0; q < VEC; q += 2) {
                        const float2 c = __fadd2_rn(make_float2(xv[q], xv[q + 1]), shift);
                        float2 u = make_float2(gv[q], gv[q + 1]);
                        if (gamma) u = __fmul2_rn(u, make_float2(wv[q], wv[q + 1]));
                        a0 = __fadd2_rn(a0, c);
                        a1 = __ffma2_rn(c, c, a1);
                        a2 = __fadd2_rn(a2, u);
                        a3 = __ffma2_rn(u, c, a3);
                    }
                }
                v[0] = a0.x + a0.y;
                v[1] = a1.x + a1.y;
                v[2] = a2.x + a2.y;
                v[3] = a3.x + a3.y;
#pragma unroll
                for (int o = 16; o > 0; o >>= 1) {
#pragma unroll
                    for (int k = 0; k < 4; ++k) v[k] += __shfl_xor_sync(0xffffffffu, v[k], o);
                }
                if (pass != 0 || !__any_sync(0xffffffffu, ln_far(v[0] * inv_d, v[1] * inv_d))) break;
                origin += v[0] * inv_d;
            }
            if (lane == 0) {
                const float off = v[0] * inv_d, um = v[2] * inv_d;
                const float sigma = sqrtf(ln_variance(off, v[1] * inv_d) + eps);
                const float rstd = 1.f / sigma;
                stat[s][0] = origin + off;
                stat[s][1] = rstd;
                stat[s][2] = um;
                stat[s][3] = fmaf(-off, um, v[3] * inv_d) * rstd;
                stat[s][4] = 1.f / fmaxf(sigma, min_rms);
                mbar_arrive(smem_u32(&ready[s]));
            }
            __syncwarp();
        }
    } else {
        // ----------------------------------------------------------------- columns
        const int t = threadIdx.x;
        P w;
        if (gamma) w.load(gamma, t, d);
        float2 dg[kSums ? kPairs : 1], db[kSums ? kPairs : 1];
#pragma unroll
        for (int i = 0; i < (kSums ? kPairs : 1); ++i) dg[i] = db[i] = both(0.f);
        int s = 0, i = 0;
        uint32_t phase = 0;
        for (; i < rows; ++i) {
            const bool in_time = ln_wait(smem_u32(&full[s]), phase, lost, limit_ns) &&
                                 ln_wait(smem_u32(&ready[s]), phase, lost, limit_ns);
            if (!__all_sync(0xffffffffu, in_time)) break;
            P xr, gr;
            xr.load(slot_x(s), t, d);
            gr.load(slot_x(s) + d, t, d);
            const float mu = stat[s][0], rstd = stat[s][1], um = stat[s][2], cm = stat[s][3],
                        pref = stat[s][4];
            __syncwarp();
            if (lane == 0) mbar_arrive(smem_u32(&empty[s]));  // all of it is in registers
            if (++s == slots) { s = 0; phase ^= 1u; }
            float2 c[kPairs], gv[kPairs], wf[kPairs];
            xr.get(c);
            gr.get(gv);
            if (gamma) w.get(wf);
            const float2 m2 = both(-mu), r2 = both(rstd), nu = both(-um), nc = both(-cm),
                         p2 = both(pref);
#pragma unroll
            for (int k = 0; k < kPairs; ++k) {
                c[k] = __fmul2_rn(__fadd2_rn(c[k], m2), r2);  // xhat
                if constexpr (kSums) {
                    dg[k] = __ffma2_rn(gv[k], c[k], dg[k]);
                    db[k] = __fadd2_rn(db[k], gv[k]);
                }
                const float2 u = gamma ? __fmul2_rn(gv[k], wf[k]) : gv[k];
                c[k] = __fmul2_rn(__ffma2_rn(c[k], nc, __fadd2_rn(u, nu)), p2);
            }
            if (out) P::store(out + ln_block_row(i) * d, t, d, c);
        }
        if (i < rows) {  // given up
            const float nan = __int_as_float(0x7fffffff);
            float2 f[kPairs];
#pragma unroll
            for (int k = 0; k < kPairs; ++k) f[k] = both(nan);
            if (out)
                for (; i < rows; ++i) P::store(out + ln_block_row(i) * d, t, d, f);
#pragma unroll
            for (int k = 0; k < (kSums ? kPairs : 1); ++k) dg[k] = db[k] = f[0];
        }
        if constexpr (kSums) {
            float* p = part + static_cast<size_t>(blockIdx.x) * 2 * d;
#pragma unroll
            for (int v = 0; v < NV; ++v) {
                const int k = (v * 32 * CW + t) * VEC;
                if (k >= d) continue;
#pragma unroll
                for (int q = 0; q < VEC; q += 2) {
                    *reinterpret_cast<float2*>(p + k + q) = dg[(v * VEC + q) / 2];
                    *reinterpret_cast<float2*>(p + d + k + q) = db[(v * VEC + q) / 2];
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
// row groups.  One cluster spares a launch and the workspace, and is slower on the GPU, which counts
// in a graph: the limit keeps that to a microsecond.  bf16 256 x 256, 4 rounds, cluster and two
// kernels: 8.2 and 15.2 us a call, 7.5 and 9.4 with a workspace of the caller's, 4.3 and 3.7 in a graph;
// 512 x 256, 8 rounds: 8.4 and 15.5, 8.3 and 9.6, but 6.5 and 4.5.
constexpr int kLnClusterRounds = 4;
bool one_cluster(int T, const RowForm& f) {
    return f.nv != 0 && f.th != 512 && T <= kLnClusterRounds * kLnCluster * (256 / f.th);
}
// Many long rows of 16-byte vectors: the stream kernels, a block to an SM.  Backward (us, stream
// kernel and register kernel): bf16 16384 x 4096 76 and 93, 16384 x 2560 70 and 87, 8192 x 8192
// 90 and 98, 300 x 4096 13 and 21; fp32 8192 x 4096 71 and 178, 16384 x 2048 74 and 76; rows of 4 KB
// come out worse (bf16 16384 x 2048 68 and 51, fp32 16384 x 1024 48 and 43), as do shorter ones
// (bf16 32768 x 1024 117 and 49).
bool streamed(int T, int d, int vec, int esz) {
    return vec > 1 && T >= 256 && d * esz > 4096 && d <= 8192;
}
// Forward: where a row leaves threads of the register kernel without elements.  bf16 8192 x 5120
// 35 and 52 us, 16384 x 2560 37 and 43, fp32 8192 x 4096 50 and 62; full ones: bf16 16384 x
// 4096 52 and 50, fp32 4096 x 8192 60 and 48; short batches: bf16 1024 x 4096 10 and 8.
bool fwd_streamed(int T, int d, int vec, int esz, const RowForm& f) {
    return T >= 4096 && d * esz > 4096 && d < f.nv * f.th * vec;
}
int stream_blocks(int T) { return T < 152 ? T : 152; }

// The form of a backward pass, and so what it needs of the workspace: one rule for both.
enum LnForm { kLongForm, kClusterForm, kStreamForm, kBlockForm };
LnForm vjp_form(int T, int d, int vec, int esz, const RowForm& f) {
    if (f.nv == 0) return kLongForm;
    if (one_cluster(T, f)) return kClusterForm;  // (without weight sums: blocks)
    return streamed(T, d, vec, esz) ? kStreamForm : kBlockForm;
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
    if constexpr (VEC > 1) {
        if (fwd_streamed(T, d, VEC, sizeof(TT), f)) {
            constexpr auto kern = layernorm_fwd_stream_kernel<TT, VEC>;
            const cudaError_t e = set_smem_limit<kern>(kLnStreamSmem);
            if (e != cudaSuccess) return e;
            const int row = d * static_cast<int>(sizeof(TT)), fit = kLnStreamSmem / row - 2;
            const int slots = fit < kLnMaxSlots ? fit : kLnMaxSlots;
            kern<<<stream_blocks(T), 32 * (kLnFwdWarps + 1), (slots + 2) * row, st>>>(
                xx, gg, bb, T, d, eps, yy, mean_out, rstd_out, slots, wait_limit_ns()),
                note_launch();
            return cudaGetLastError();
        }
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
    const LnForm form = vjp_form(T, d, VEC, sizeof(TT), f);
    int parts = 0;
    cudaError_t e;
    if (form == kLongForm) {
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
    } else if (form == kStreamForm) {
        if constexpr (VEC > 1) {
            parts = stream_blocks(T);
            auto launch = [&](auto nv, auto cw, auto sw, auto mode) {
                constexpr int CW = decltype(cw)::value, SW = decltype(sw)::value;
                using S = LnStream<CW, SW>;
                constexpr auto kern = layernorm_vjp_stream_kernel<TT, VEC, decltype(nv)::value, CW, SW,
                                                                  decltype(mode)::value != 0>;
                const cudaError_t le = set_smem_limit<kern>(kLnStreamSmem);
                if (le != cudaSuccess) return le;
                const int row = d * static_cast<int>(sizeof(TT)), fit = (kLnStreamSmem - row) / (2 * row);
                const int slots = fit < kLnMaxSlots ? fit : kLnMaxSlots;
                kern<<<parts, S::kThreads, (2 * slots + 1) * row, st>>>(
                    gg, xx, ww, T, d, eps, min_rms, oo, ws, slots, wait_limit_ns()),
                    note_launch();
                return cudaGetLastError();
            };
            auto run = [&](auto nv, auto cw, auto sw) {
                return sums ? launch(nv, cw, sw, Int<1>{}) : launch(nv, cw, sw, Int<0>{});
            };
            const int n = d / VEC;
            if constexpr (VEC == 4)
                e = n <= 512    ? run(Int<2>{}, Int<8>{}, Int<8>{})
                    : n <= 1024 ? run(Int<4>{}, Int<8>{}, Int<8>{})
                                : run(Int<4>{}, Int<16>{}, Int<3>{});
            else
                e = n <= 512 ? run(Int<2>{}, Int<8>{}, Int<8>{}) : run(Int<2>{}, Int<16>{}, Int<7>{});
        } else {
            e = cudaErrorInvalidValue;  // (streamed)
        }
    } else if (form == kClusterForm && sums) {
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
    const int vec = dtype == 1 ? 8 : d % 4 == 0 ? 4 : 1;
    const RowForm f = vec == 8   ? row_form<__nv_bfloat16, 8>(d)
                      : vec == 4 ? row_form<float, 4>(d)
                                 : row_form<float, 1>(d);
    const size_t sums = 2 * static_cast<size_t>(d);
    switch (vjp_form(T, d, vec, dtype == 1 ? 2 : 4, f)) {
        case kLongForm: return 2 * static_cast<size_t>(T) + long_ranges(T) * sums;
        case kClusterForm: return 0;
        case kStreamForm: return stream_blocks(T) * sums;
        default: return vjp_blocks(T, f) * sums;
    }
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
