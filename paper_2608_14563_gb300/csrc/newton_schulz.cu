// newton_schulz.cu -- orthogonalised updates: K steps of an odd quintic iteration on the
// matrix of every layer, and the optimizer step that takes them (the orthogonalised momentum
// of the Muon optimizer on the fp32 masters of Sec. 3.1).
//
//   X_0 = G / max(||G||_F, eps)                 singular values in [0, 1]
//   X_{k+1} = a X_k + (b A + c A^2) X_k,  A = X_k X_k^T     p_k(s) = a s + b s^3 + c s^5
//
// (X (b A + c A^2) with A = X^T X when X is taller than wide: the products of the smaller
// side).  Per step m^2 n + m^3 + 2 m^2 n operations for sides m <= n, the first two halved by
// symmetry; bound by the tensor cores for all but small matrices.
//
// Number formats.  Operands are fp16 (11 bits; bf16's 8 leave 1e-2 of error in the result)
// scaled by powers of two: the host bounds every X_k, A and B from the polynomials' maxima on
// the interval that the singular values can reach, so nothing overflows, and fp16's small end
// lies 2^-39 below the bound.  bf16 calls keep X's low part for the linear term (EpiApply);
// against fp64 their result is then off by 0.7e-3 to 2.0e-3 in norm before its own rounding
// (1.7e-3), whatever the rank.  fp32 calls, and bf16 ones of few rows or columns (ns_split), take
// every operand as the sum of two fp16 matrices (22 bits) and three products: 1e-6 to 2e-6.
//
// Launches: norm, cast, then A, B, X' of every step (in one launch where few tiles make its
// waits cheaper than launches, ns_chain_kernel).  4096 x 11008, five steps (us, one launch each,
// alone): norm 29, cast 46, A 118, B 51, X' 242 (last 218): the products at 70 to 84% of the tensor
// rate in whole waves of tiles on 76 clusters, 136 tiles of A taking two and the 688 of X' ten.
// Muon: the gradient's GEMM with the momentum and the squares in its epilogue, and a last pass
// over the masters at the copy rate (4096 x 11008 twice, 4096 tokens: 536 and 189 us).
#include <cuda.h>
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <math.h>

#include <atomic>
#include <mutex>

#include "internal.h"
#include "ns_gemm.cuh"

namespace fpo {
namespace {

constexpr int kPassThreads = 256;
constexpr int kNormBlocks = 304;  // per layer, at most: 2 on each of 152 SMs

struct NsPtrs {
    const void* in[kMaxGroups];  // G, or U (fp32)
    float* M[kMaxGroups];        // momentum, or null
};

__device__ __forceinline__ double block_sum_d(double x) {
    __shared__ double sh[kPassThreads / 32];
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
    if ((threadIdx.x & 31) == 0) sh[threadIdx.x >> 5] = x;
    __syncthreads();
    double t = 0.0;
#pragma unroll
    for (int k = 0; k < kPassThreads / 32; ++k) t += sh[k];
    return t;
}

// Sum of the squares of 16 values: fp32 where that neither overflows nor loses digits to
// underflow, else fp64 (GB300 adds two fp64 numbers per SM and clock).
__device__ __forceinline__ double square_sum16(const float (&v)[16]) {
    float s = 0.f;
#pragma unroll
    for (int k = 0; k < 16; ++k) s = fmaf(v[k], v[k], s);
    if (s >= 1e-30f && s <= 3e38f) return s;
    uint32_t any = 0;  // zeros are frequent, and need no fp64
#pragma unroll
    for (int k = 0; k < 16; ++k) any |= __float_as_uint(v[k]) << 1;
    if (any == 0) return 0.0;
    double d = 0.0;
#pragma unroll
    for (int k = 0; k < 16; ++k) d += static_cast<double>(v[k]) * v[k];
    return d;
}

// 16 consecutive elements of an array of n, zeros behind its end.  16-byte aligned base.
__device__ __forceinline__ void load16(const float* p, size_t i, size_t n, float (&v)[16]) {
    if (i + 16 <= n) {
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const float4 a = reinterpret_cast<const float4*>(p + i)[k];
            v[4 * k] = a.x;
            v[4 * k + 1] = a.y;
            v[4 * k + 2] = a.z;
            v[4 * k + 3] = a.w;
        }
    } else {
#pragma unroll
        for (int k = 0; k < 16; ++k) v[k] = i + k < n ? p[i + k] : 0.f;
    }
}
__device__ __forceinline__ void load16(const __nv_bfloat16* p, size_t i, size_t n, float (&v)[16]) {
    if (i + 16 <= n) {
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            const uint4 a = reinterpret_cast<const uint4*>(p + i)[k];
            const uint32_t w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                v[8 * k + 2 * j] = __uint_as_float(w[j] << 16);
                v[8 * k + 2 * j + 1] = __uint_as_float(w[j] & 0xffff0000u);
            }
        }
    } else {
#pragma unroll
        for (int k = 0; k < 16; ++k) v[k] = i + k < n ? __bfloat162float(p[i + k]) : 0.f;
    }
}
__device__ __forceinline__ void store16(float* p, size_t i, size_t n, const float (&v)[16]) {
    if (i + 16 <= n) {
#pragma unroll
        for (int k = 0; k < 4; ++k)
            reinterpret_cast<float4*>(p + i)[k] =
                make_float4(v[4 * k], v[4 * k + 1], v[4 * k + 2], v[4 * k + 3]);
    } else {
#pragma unroll
        for (int k = 0; k < 16; ++k)
            if (i + k < n) p[i + k] = v[k];
    }
}

__device__ __forceinline__ void store16(__nv_bfloat16* p, size_t i, size_t n, const float (&v)[16]) {
    if (i + 16 <= n) {
        uint32_t w[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) w[k] = pack_bf16x2(v[2 * k], v[2 * k + 1]);
        reinterpret_cast<uint4*>(p + i)[0] = make_uint4(w[0], w[1], w[2], w[3]);
        reinterpret_cast<uint4*>(p + i)[1] = make_uint4(w[4], w[5], w[6], w[7]);
    } else {
#pragma unroll
        for (int k = 0; k < 16; ++k)
            if (i + k < n) p[i + k] = __float2bfloat16_rn(v[k]);
    }
}

// part[layer][block] = sum of squares over the block's share of the layer's n elements.
template <typename TT>
__global__ void __launch_bounds__(kPassThreads)
    ns_norm_kernel(const __grid_constant__ NsPtrs p, size_t n, double* part) {
    grid_dependency_trigger();
    grid_dependency_wait();
    const int layer = blockIdx.y;
    const size_t step = static_cast<size_t>(gridDim.x) * kPassThreads * 16;
    double acc = 0.0;
    const TT* src = static_cast<const TT*>(p.in[layer]);
    for (size_t i = (blockIdx.x * static_cast<size_t>(kPassThreads) + threadIdx.x) * 16; i < n;
         i += 4 * step) {
        float v[4][16];
#pragma unroll
        for (int q = 0; q < 4; ++q) load16(src, i + q * step, n, v[q]);
#pragma unroll
        for (int q = 0; q < 4; ++q) acc += square_sum16(v[q]);
    }
    const double t = block_sum_d(acc);
    if (threadIdx.x == 0) part[static_cast<size_t>(layer) * gridDim.x + blockIdx.x] = t;
}

// The momentum: M <- mu M + G and U = G + mu M (nesterov) or M, U over G; sums of the squares of
// U as ns_norm_kernel leaves them.  (Launched plainly, behind the gradient's GEMM.)
__global__ void __launch_bounds__(kPassThreads)
    ns_momentum_kernel(const __grid_constant__ NsPtrs p, size_t n, float mu, bool nesterov,
                       double* part) {
    const int layer = blockIdx.y;
    float* U = static_cast<float*>(const_cast<void*>(p.in[layer]));
    float* M = p.M[layer];
    const size_t step = static_cast<size_t>(gridDim.x) * kPassThreads * 16;
    double acc = 0.0;
    for (size_t i = (blockIdx.x * static_cast<size_t>(kPassThreads) + threadIdx.x) * 16; i < n;
         i += step) {
        float v[16], m[16];
        load16(U, i, n, v);
        load16(M, i, n, m);
#pragma unroll
        for (int k = 0; k < 16; ++k) {
            m[k] = fmaf(mu, m[k], v[k]);
            v[k] = nesterov ? fmaf(mu, m[k], v[k]) : m[k];
        }
        store16(M, i, n, m);
        store16(U, i, n, v);
        acc += square_sum16(v);
    }
    const double t = block_sum_d(acc);
    if (threadIdx.x == 0) part[static_cast<size_t>(layer) * gridDim.x + blockIdx.x] = t;
}

// W <- keep W - rate O, and out (or null) = W in the call's type; neither where a wait of the call
// has run out, for O is then no result.  A pass of its own: 12 to 18 bytes an element.
struct NsWeights {
    const float* O[kMaxGroups];
    float* W[kMaxGroups];
    void* out[kMaxGroups];
};

template <typename TT>
__global__ void __launch_bounds__(kPassThreads)
    ns_weight_kernel(const __grid_constant__ NsWeights p, size_t n, float keep, float rate,
                     const unsigned* status) {
    grid_dependency_trigger();
    grid_dependency_wait();
    if (*status != 0) return;
    const int layer = blockIdx.y;
    const float* O = p.O[layer];
    float* W = p.W[layer];
    TT* out = static_cast<TT*>(p.out[layer]);
    const size_t step = static_cast<size_t>(gridDim.x) * kPassThreads * 16;
    for (size_t i = (blockIdx.x * static_cast<size_t>(kPassThreads) + threadIdx.x) * 16; i < n;
         i += step) {
        float v[16], w[16];
        load16(O, i, n, v);
        load16(W, i, n, w);
#pragma unroll
        for (int k = 0; k < 16; ++k) w[k] = fmaf(-rate, v[k], keep * w[k]);
        store16(W, i, n, w);
        if (out) store16(out, i, n, w);
    }
}

// sum[layer] of the layer's `blocks` partial sums, in a fixed order.
constexpr int kSumThreads = 1024;
__global__ void __launch_bounds__(kSumThreads)
    ns_sum_kernel(const double* part, int blocks, double* sum) {
    __shared__ double sh[kSumThreads / 32];
    grid_dependency_trigger();
    grid_dependency_wait();
    const double* p = part + static_cast<size_t>(blockIdx.x) * blocks;
    double x = 0.0;
    for (int b = threadIdx.x; b < blocks; b += kSumThreads) x += p[b];
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
    if ((threadIdx.x & 31) == 0) sh[threadIdx.x >> 5] = x;
    __syncthreads();
    if (threadIdx.x >= 32) return;
    x = sh[threadIdx.x];
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
    if (threadIdx.x == 0) sum[blockIdx.x] = x;
}

// scale / max(sqrt(s), eps) in fp32 arithmetic (fp64 roots and quotients take microseconds here);
// NaN if s is not finite.
__device__ __forceinline__ float norm_factor(double s, float scale, float eps) {
    const long long bits = __double_as_longlong(s);
    const int e = static_cast<int>((bits >> 52) & 0x7ff) - 1023;  // s = m 2^e
    if (e == 1024) return NAN;
    if (e == -1023) return scale / eps;  // zero
    const int h = e >> 1;  // s = (m 2^(e - 2 h)) 4^h, the bracket in [1, 4)
    const float r = sqrtf(static_cast<float>(__longlong_as_double(
        (bits & 0x000fffffffffffffll) | (static_cast<long long>(1023 + e - 2 * h) << 52))));
    return ldexpf(r, h) < eps ? scale / eps : ldexpf(scale / r, -h);
}

// X_0, scaled: fp16 high and low parts (kSplit: and the fp32 value), rows ld apart.  Thread: 8
// columns of a row (what it writes past cols is never read: the tensor maps end at cols, and a
// linear term past them goes nowhere).  The layer's norm from its `blocks` partial sums.
// A layer with a non-finite norm (a NaN, an infinity) becomes NaN as a whole.
template <typename TT, bool kSplit>
__global__ void __launch_bounds__(kPassThreads)
    ns_cast_kernel(const __grid_constant__ NsPtrs p, int rows, int cols, int ld, const double* part,
                   int blocks, float eps, float scale, __half* hi, __half* lo, float* x32,
                   size_t stride) {
    grid_dependency_trigger();
    grid_dependency_wait();
    const int layer = blockIdx.y;
    double s = 0.0;
    for (int b = threadIdx.x; b < blocks; b += kPassThreads)
        s += part[static_cast<size_t>(layer) * blocks + b];
    const float f = norm_factor(block_sum_d(s), scale, eps);
    const TT* src = static_cast<const TT*>(p.in[layer]);
    const int per = (cols + 7) / 8;
    const bool vec = cols % 8 == 0;  // rows then start on 16 bytes
    const size_t n = static_cast<size_t>(rows) * per;
    for (size_t i = blockIdx.x * static_cast<size_t>(kPassThreads) + threadIdx.x; i < n;
         i += static_cast<size_t>(gridDim.x) * kPassThreads) {
        const size_t row = i / per;
        const int col = static_cast<int>(i - row * per) * 8;
        const TT* q = src + row * cols + col;
        float v[8];
        if (vec) {
            if constexpr (sizeof(TT) == 2) {
                const uint4 a = *reinterpret_cast<const uint4*>(q);
                const uint32_t w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    v[2 * j] = __uint_as_float(w[j] << 16);
                    v[2 * j + 1] = __uint_as_float(w[j] & 0xffff0000u);
                }
            } else {
                const float4 a = reinterpret_cast<const float4*>(q)[0];
                const float4 b = reinterpret_cast<const float4*>(q)[1];
                v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w;
                v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
            }
        } else {
#pragma unroll
            for (int k = 0; k < 8; ++k) v[k] = col + k < cols ? static_cast<float>(q[k]) : 0.f;
        }
        uint32_t h[4], l[4];
#pragma unroll
        for (int k = 0; k < 8; ++k) v[k] *= f;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            h[k] = pack_f16x2(v[2 * k], v[2 * k + 1]);
            const float2 g = unpack_f16x2(h[k]);
            l[k] = pack_f16x2(v[2 * k] - g.x, v[2 * k + 1] - g.y);
        }
        const size_t o = layer * stride + row * ld + col;
        *reinterpret_cast<uint4*>(hi + o) = make_uint4(h[0], h[1], h[2], h[3]);
        *reinterpret_cast<uint4*>(lo + o) = make_uint4(l[0], l[1], l[2], l[3]);
        if constexpr (kSplit) {
            reinterpret_cast<float4*>(x32 + o)[0] = make_float4(v[0], v[1], v[2], v[3]);
            reinterpret_cast<float4*>(x32 + o)[1] = make_float4(v[4], v[5], v[6], v[7]);
        }
    }
}

size_t round_up(size_t x, size_t m) { return (x + m - 1) / m * m; }

int norm_blocks(size_t n) {
    const size_t b = (n + kPassThreads * 16 - 1) / (kPassThreads * 16);
    return static_cast<int>(b < kNormBlocks ? b : kNormBlocks);
}

// Partial sums of squares of one layer: a block's of the norm pass, or a warp's of a tile of the
// gradient's GEMM (of at most 256 x 128).
size_t norm_parts(int rows, int cols, bool muon) {
    const size_t tiles = static_cast<size_t>((rows + 255) / 256) * ((cols + 127) / 128);
    const size_t slots = muon ? tiles * 2 * kNsWarps : 0;
    return slots > kNormBlocks ? slots : kNormBlocks;
}

// Byte offsets of the workspace behind the status word's 256 bytes.
struct NsLayout {
    int m, ld, ldm;              // the smaller side, row strides of X and of A, B
    size_t xs, ms;               // elements of one layer's X, A
    size_t counts, slots;        // split: of the ranges of A = X X^T (NsShape)
    size_t part, sum, U, u_stride, hi[2], lo[2], x32, A[2], B[2], total;
    size_t clear;                // bytes from the start to be zero before a call
};

// Tiles of one matrix of a kSplit product [M, N], and the ranges that the k-blocks of A = X X^T
// (X^T X) are split into: as many as half of the 76 clusters hold of one matrix, of 16 k-blocks or
// more.  (For A^2 and X', whose k is the smaller side, the same rule would never give two: 32 k-blocks
// are 72 tiles or more.)  It goes by the matrix's sizes only, so that its result does not depend on
// the group.  Five steps, with and without: 767 x 2049 one matrix 314 and 349 us, two 380 and 413,
// eight 977 and 944; eight 256 x 4096 388 and 510, eight 512 x 2048 580 and 525; two 64 x 8192 231
// and 555.  (Ranges of 8 k-blocks: eight 512 x 1024 392 instead of 332.)
long long ns_matrix_tiles(int M, int N, bool tri) {
    const long long mb = (M + 255) / 256;
    return tri ? mb * (mb + 1) : mb * ((N + 127) / 128);
}
int ns_splits(long long tiles, int K) {
    const long long clusters = 38 / tiles, blocks = (K + kBK - 1) / kBK / 16;
    const long long s = clusters < blocks ? clusters : blocks;
    return s < 1 ? 1 : static_cast<int>(s);
}

// kSplit: fp32 calls, and bf16 ones of few rows or columns: there the rounding errors of single
// entries of A and B average out least.  In norm the bf16 result of fp16 products is off by 2.3e-3 to
// 3.9e-3 for sides of 8 to 64, 2.0e-3 to 2.6e-3 for longer ones (its own rounding, and all of
// it with kSplit: 1.7e-3).  Two 64 x 256 matrices take 121 us instead of 83, sixteen 64 x 4096
// 399 instead of 280, one 16 x 8192 200 instead of 239.
bool ns_split(int dtype, int rows, int cols) {
    return dtype == 0 || rows <= 64 || cols <= 64;
}

NsLayout ns_layout(int n, int rows, int cols, int dtype, bool muon) {
    const bool split = ns_split(dtype, rows, cols);
    NsLayout L = {};
    L.m = rows < cols ? rows : cols;
    // rows of whole 128-byte lines: a TMA box of 64 columns then takes one line of a row, not two
    // (fp32 767 x 2049, two matrices: 510 us with rows of 16-byte multiples, 487 with these)
    L.ld = static_cast<int>(round_up(cols, 64));
    L.ldm = static_cast<int>(round_up(L.m, 64));
    L.xs = static_cast<size_t>(rows) * L.ld;
    L.ms = static_cast<size_t>(L.m) * L.ldm;
    L.u_stride = round_up(static_cast<size_t>(rows) * cols, 64);
    size_t at = 256;
    auto take = [&](size_t bytes) {
        const size_t o = at;
        at += round_up(bytes, 256);
        return o;
    };
    L.clear = 2 * sizeof(unsigned);  // the status word and the chain kernel's counter
    if (split) {
        const long long tiles = ns_matrix_tiles(L.m, L.m, true);
        const long long ranges = ns_splits(tiles, rows < cols ? cols : rows);
        if (ranges > 1) {
            L.counts = take(n * tiles * 2 * kNsWarps * sizeof(unsigned));
            L.clear = at;
            L.slots = take(n * tiles * ranges * (kPairBM * 128 * sizeof(float)));
        }
    }
    const size_t x = n * L.xs * 2, a = n * L.ms * 2;
    L.part = take(static_cast<size_t>(n) * norm_parts(rows, cols, muon) * sizeof(double));
    L.sum = take(static_cast<size_t>(n) * sizeof(double));
    L.U = muon ? take(n * L.u_stride * 4) : 0;
    L.hi[0] = take(x);
    L.hi[1] = take(x);
    L.lo[0] = take(x);
    L.lo[1] = split ? take(x) : L.lo[0];  // a linear term's low part is updated in place
    L.x32 = split ? take(2 * x) : 0;
    L.A[0] = take(a);
    L.B[0] = take(a);
    L.A[1] = split ? take(a) : 0;
    L.B[1] = split ? take(a) : 0;
    L.total = at;
    return L;
}

using EncodeTiledFn = CUresult (*)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*,
                                   const cuuint64_t*, const cuuint64_t*, const cuuint32_t*,
                                   const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle,
                                   CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

EncodeTiledFn encode_fn() {
    static EncodeTiledFn fn = nullptr;
    static std::once_flag once;
    std::call_once(once, [] {
        void* p = nullptr;
        cudaDriverEntryPointQueryResult q;
        if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &p, 12000, cudaEnableDefault,
                                             &q) == cudaSuccess &&
            q == cudaDriverEntryPointSuccess)
            fn = reinterpret_cast<EncodeTiledFn>(p);
    });
    return fn;
}

// A batch [n][outer][inner] of fp16 matrices (row stride ld, matrix stride `stride` elements), the
// high and (kSplit) low parts.
struct NsOperand {
    const __half* p[2];
    int inner, outer, n, ld;
    size_t stride;
};

// One part as a GEMM operand: K-major (inner = k: boxes of 64 k x `rows` rows) or MN-major (64
// columns x 64 k); 128-byte swizzle, zeros outside each matrix.
bool ns_map(CUtensorMap* m, const NsOperand& o, int part, bool mn, int rows,
            CUtensorMapDataType type = CU_TENSOR_MAP_DATA_TYPE_FLOAT16) {
    const EncodeTiledFn fn = encode_fn();
    if (!fn) return false;
    cuuint64_t dims[3] = {static_cast<cuuint64_t>(o.inner), static_cast<cuuint64_t>(o.outer),
                          static_cast<cuuint64_t>(o.n)};
    cuuint64_t strides[2] = {static_cast<cuuint64_t>(o.ld) * 2, o.stride * 2};
    cuuint32_t box[3] = {64, mn ? 64u : static_cast<cuuint32_t>(rows), 1};
    cuuint32_t es[3] = {1, 1, 1};
    return fn(m, type, 3, const_cast<__half*>(o.p[part]), dims, strides, box, es,
              CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
              CU_TENSOR_MAP_L2_PROMOTION_L2_128B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// Pair clusters of a kernel that can be resident at once on the current device, computed once
// per device (after the kernel's shared-memory limit is raised there).
template <auto Kern>
int resident_clusters(int threads, int smem_bytes, int sm_count) {
    static std::atomic<int> cache[kMaxDevices];
    const int dev = current_device();
    if (dev < 0) return sm_count / 2;
    int n = cache[dev].load(std::memory_order_relaxed);
    if (n > 0) return n;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(static_cast<unsigned>(sm_count / 2 * 2), 1, 1);
    cfg.blockDim = dim3(static_cast<unsigned>(threads), 1, 1);
    cfg.dynamicSmemBytes = static_cast<size_t>(smem_bytes);
    if (cudaOccupancyMaxActiveClusters(&n, Kern, &cfg) != cudaSuccess || n < 1) {
        cudaGetLastError();
        n = sm_count / 2;
    }
    cache[dev].store(n, std::memory_order_relaxed);
    return n;
}

// Where the ranges of A = X X^T leave their sums (kSplit; null: no ranges).
struct NsRanges {
    float* slots;
    unsigned* counts;
};

template <int BN, bool A_MN, bool B_MN, bool kSplit, class Epi>
cudaError_t launch_ns(const typename Epi::Maps& maps, const typename Epi::Params& ep, int M, int N,
                      int K, int groups, bool tri, const NsRanges& rg, unsigned* status,
                      cudaStream_t st) {
    using S = NsSmem<BN>;
    constexpr auto kern = ns_gemm_kernel<BN, A_MN, B_MN, kSplit, Epi>;
    cudaError_t e = set_smem_limit<kern>(S::kBytes);
    if (e != cudaSuccess) return e;
    DevInfo di;
    if (!current_device_info(&di)) return cudaErrorUnknown;
    NsShape sh = {};
    sh.tri = tri;
    sh.g.M = M;
    sh.g.N = N;
    sh.g.K = K;
    sh.g.m_blocks = (M + kPairBM - 1) / kPairBM;
    sh.g.n_blocks = (N + BN - 1) / BN;
    sh.g.k_blocks = (K + kBK - 1) / kBK;
    sh.g.groups = groups;
    sh.g.band = 16;
    const long long per =
        tri ? static_cast<long long>(sh.g.m_blocks) * (sh.g.m_blocks + 1) / 2 * (kPairBM / BN)
            : static_cast<long long>(sh.g.m_blocks) * sh.g.n_blocks;
    sh.g.tiles = groups * per;
    sh.splits = Epi::kRanges && rg.slots ? ns_splits(ns_matrix_tiles(M, N, tri), K) : 1;
    sh.slots = rg.slots;
    sh.counts = rg.counts;
    constexpr int kThreads = ns_threads<BN, kSplit, Epi>();
    if constexpr (ns_first_warp<BN, kSplit, Epi>() == 4) {
        // the warpgroups' new shares have to fit into what the block is launched with: an increase
        // beyond it would never be granted
        static std::atomic<int> regs{0};
        if (regs.load(std::memory_order_relaxed) == 0) {
            cudaFuncAttributes at;
            e = cudaFuncGetAttributes(&at, kern);
            if (e != cudaSuccess) return e;
            regs.store(at.numRegs, std::memory_order_relaxed);
        }
        if (regs.load(std::memory_order_relaxed) * kThreads < 128 * (kNsFewRegs + 2 * kNsManyRegs))
            return cudaErrorLaunchOutOfResources;
    }
    const int max_clusters = resident_clusters<kern>(kThreads, S::kBytes, di.sm_count);
    const long long units = sh.g.tiles * sh.splits;
    const long long clusters = units < max_clusters ? units : max_clusters;
    return launch_chained(kern, dim3(static_cast<unsigned>(2 * clusters)), kThreads, S::kBytes, st, maps,
                          ep, sh, status, wait_limit_ns());
}

// One batch of GEMMs, C[M, N] = sum_k A B over K, on the pair kernel with 256 x BN tiles.
template <int BN, bool A_MN, bool B_MN, bool kSplit, class Epi>
cudaError_t run_ns_tiles(const NsOperand& A, const NsOperand& B, const typename Epi::Params& ep,
                         int M, int N, int K, bool tri, const NsRanges& rg, unsigned* status,
                         cudaStream_t st) {
    NsMaps maps;
    for (int h = 0; h < 2; ++h) {
        if (h == 1 && !kSplit) {
            maps.a[1] = maps.a[0];
            maps.b[1] = maps.b[0];
        } else if (!ns_map(&maps.a[h], A, h, A_MN, 128) || !ns_map(&maps.b[h], B, h, B_MN, BN / 2)) {
            return cudaErrorInvalidValue;
        }
    }
    return launch_ns<BN, A_MN, B_MN, kSplit, Epi>(maps, ep, M, N, K, A.n, tri, rg, status, st);
}

// Tiles of 256 columns or of 128 (the same bits).  fp16: 128 where twice as many tiles still have a
// cluster each, an epilogue is then half as long.  kSplit, whose epilogue no MMAs hide, by the waves
// of tiles on the clusters times a tile's time: 1.03 us a 64-deep k-block and 12 us of set-up and
// epilogue with 256 columns, 0.85 and 4 with 128.  (Five steps, 128 columns alone and by this rule:
// one 2048 x 8192 1636 and 1475 us, two 767 x 2049 380 and 355, eight 512 x 1024 332 and 321;
// 256 wherever fp16 takes them: eight 256 x 4096 405 instead of 381.)
template <bool A_MN, bool B_MN, bool kSplit, template <int> class Epi>
cudaError_t run_ns(const NsOperand& A, const NsOperand& B, const typename Epi<128>::Params& ep, int M,
                   int N, int K, bool tri, const NsRanges& rg, unsigned* status, cudaStream_t st) {
    DevInfo di;
    if (!current_device_info(&di)) return cudaErrorUnknown;
    const long long mb = (M + 255) / 256, nb = (N + 255) / 256;
    const long long tiles = A.n * (tri ? mb * (mb + 1) / 2 : mb * nb);
    bool wide = 4 * tiles > di.sm_count;
    if constexpr (kSplit) {
        const long long narrow = ns_matrix_tiles(M, N, tri), clusters = di.sm_count / 2;
        const int splits = rg.slots ? ns_splits(narrow, K) : 1, blocks = (K + kBK - 1) / kBK / splits;
        auto waves = [&](long long units) { return (units + clusters - 1) / clusters; };
        wide = waves(tiles * splits) * (1030 * blocks + 12000) <
               waves(A.n * narrow * splits) * (850 * blocks + 4000);
    }
    if (wide)
        return run_ns_tiles<256, A_MN, B_MN, kSplit, Epi<256>>(A, B, ep, M, N, K, tri, rg, status, st);
    return run_ns_tiles<128, A_MN, B_MN, kSplit, Epi<128>>(A, B, ep, M, N, K, tri, rg, status, st);
}

template <bool kSplit>
struct SymOf {
    template <int BN>
    using T = EpiSym<BN, kSplit>;
};
template <bool kSplit, int kOut>
struct ApplyOf {
    template <int BN>
    using T = EpiApply<BN, kSplit, kOut>;
};

// Largest |c1 s + c3 s^3 + c5 s^5| (odd) on [0, u].
double odd_max(double c1, double c3, double c5, double u) {
    double best = fabs(u * (c1 + u * u * (c3 + u * u * c5)));
    auto at = [&](double z) {  // z = s^2 of a critical point
        if (z > 0.0 && z < u * u) {
            const double s = sqrt(z);
            const double v = fabs(s * (c1 + z * (c3 + z * c5)));
            if (v > best) best = v;
        }
    };
    // The roots of c1 + 3 c3 z + 5 c5 z^2 as h / (5 c5) and c1 / h, h = -(3 c3 +- sqrt(..)) / 2 with
    // the sign that adds: neither is lost to cancellation, however small c5 or c1 is.
    const double q = 9.0 * c3 * c3 - 20.0 * c5 * c1;
    if (q >= 0.0) {
        const double h = -0.5 * (3.0 * c3 + copysign(sqrt(q), c3));
        if (c5 != 0.0) at(h / (5.0 * c5));
        if (h != 0.0) at(c1 / h);
    }
    return best;
}

// Largest |b t + c t^2| on [0, t1].
double quad_max(double b, double c, double t1) {
    double best = fabs(t1 * (b + c * t1));
    if (c != 0.0) {
        const double t = -b / (2.0 * c);
        if (t > 0.0 && t < t1) best = fmax(best, fabs(t * (b + c * t)));
    }
    return best;
}

// The power of two that brings a bound to at most 2^15, half of fp16's largest value: what
// rounding adds to a bound stays far below the other half.
int scale_exp(double bound) { return 15 - static_cast<int>(ceil(log2(bound))); }

NsRanges ns_ranges(const NsLayout& L, uint8_t* ws) {
    if (L.slots == 0) return {};
    return {reinterpret_cast<float*>(ws + L.slots), reinterpret_cast<unsigned*>(ws + L.counts)};
}

// X' = a X + B X (tall: a X + X B) and what becomes of it; ep holds the coefficients and targets.
template <bool kSplit, int kOut>
cudaError_t run_apply(const NsOperand& X, const NsOperand& B, bool tall, const NsLayout& L, uint8_t* ws,
                      int cur, bool next_lo, typename EpiApplyBase<kSplit, kOut>::Params& ep,
                      unsigned* status, cudaStream_t st) {
    const int rows = X.outer, cols = X.inner;
    ep.s.hi = X.p[0];
    ep.s.lo = reinterpret_cast<__half*>(ws + L.lo[cur]);
    ep.s.next_hi = reinterpret_cast<__half*>(ws + L.hi[cur ^ 1]);
    ep.s.next_lo = next_lo ? reinterpret_cast<__half*>(ws + L.lo[cur ^ 1]) : nullptr;
    ep.x32 = kSplit ? reinterpret_cast<float*>(ws + L.x32) : nullptr;
    ep.stride = static_cast<long long>(L.xs);
    ep.M = rows;
    ep.N = cols;
    ep.ld = L.ld;
    // wide: B X with B K-major and X MN-major; tall: X B, both K-major (B is symmetric)
    if (tall)
        return run_ns<false, false, kSplit, ApplyOf<kSplit, kOut>::template T>(X, B, ep, rows, cols,
                                                                              cols, false, {}, status,
                                                                              st);
    return run_ns<false, true, kSplit, ApplyOf<kSplit, kOut>::template T>(B, X, ep, rows, cols, rows,
                                                                         false, {}, status, st);
}

// The coefficients of every product with the powers of two that X, A and B are stored with: X_k
// times 2^sx (2^15 for X_0, 1 for the result), A times 2^sa, B times 2^sb.
void ns_steps(int steps, const float* coeffs, NsChainStep* out) {
    double u = 1.0;            // bound of the singular values of X_k
    int sx = scale_exp(u);
    for (int k = 0; k < steps; ++k) {
        const double a = coeffs[3 * k], b = coeffs[3 * k + 1], c = coeffs[3 * k + 2];
        const double ub = quad_max(b, c, u * u), un = odd_max(a, b, c, u);
        const int sa = scale_exp(u * u), sb = ub > 0.0 ? scale_exp(ub) : 0,
                  sn = k == steps - 1 ? 0 : scale_exp(un);
        out[k].a_acc = static_cast<float>(ldexp(1.0, sa - 2 * sx));
        out[k].b_lin = static_cast<float>(ldexp(b, sb - sa));
        out[k].b_acc = static_cast<float>(ldexp(c, sb - 2 * sa));
        out[k].x_lin = static_cast<float>(ldexp(a, sn - sx));
        out[k].x_acc = static_cast<float>(ldexp(1.0, sn - sb - sx));
        u = un;
        sx = sn;
    }
}

template <bool kSplit, int kOut>
void set_target(typename EpiApplyBase<kSplit, kOut>::Params& ep, int n, void* const* O) {
    using Out = typename EpiApplyBase<kSplit, kOut>::Out;
    for (int l = 0; l < n; ++l) ep.out[l] = static_cast<Out*>(O[l]);
}

// The iteration on the X_0 in the workspace, a launch per product.  The last step takes the
// linear term of fp16 calls from the operand itself: nothing grows after it, and the same X in
// both terms is the smaller error.
template <bool kSplit, int kOut>
cudaError_t run_steps(const NsLayout& L, uint8_t* ws, int n, int rows, int cols, int steps,
                      const NsChainStep* co, void* const* O, unsigned* status, cudaStream_t st) {
    const bool tall = rows > cols;
    const NsRanges rg = ns_ranges(L, ws);
    auto at = [&](size_t off) { return reinterpret_cast<__half*>(ws + off); };
    const NsOperand A = {{at(L.A[0]), at(L.A[1])}, L.m, L.m, n, L.ldm, L.ms};
    const NsOperand B = {{at(L.B[0]), at(L.B[1])}, L.m, L.m, n, L.ldm, L.ms};
    int cur = 0;
    for (int k = 0; k < steps; ++k) {
        const NsOperand X = {{at(L.hi[cur]), at(L.lo[cur])}, cols, rows, n, L.ld, L.xs};
        // A = X X^T
        typename EpiSymBase<kSplit>::Params sp = {};
        sp.stride = static_cast<long long>(L.ms);
        sp.M = L.m;
        sp.ld = L.ldm;
        sp.out[0] = at(L.A[0]);
        sp.out[1] = at(L.A[1]);
        sp.acc_coef = co[k].a_acc;
        cudaError_t e = tall ? run_ns<true, true, kSplit, SymOf<kSplit>::template T>(
                                   X, X, sp, L.m, L.m, rows, true, rg, status, st)
                             : run_ns<false, false, kSplit, SymOf<kSplit>::template T>(
                                   X, X, sp, L.m, L.m, cols, true, rg, status, st);
        if (e != cudaSuccess) return e;
        // B = b A + c A^2
        sp.lin[0] = at(L.A[0]);
        sp.lin[1] = at(L.A[1]);
        sp.out[0] = at(L.B[0]);
        sp.out[1] = at(L.B[1]);
        sp.lin_coef = co[k].b_lin;
        sp.acc_coef = co[k].b_acc;
        e = run_ns<false, false, kSplit, SymOf<kSplit>::template T>(A, A, sp, L.m, L.m, L.m, true, {},
                                                                    status, st);
        if (e != cudaSuccess) return e;
        // X' = a X + B X
        const bool last = k == steps - 1;
        auto coefs = [&](NsApplyStep& s) {
            s.lin_coef = co[k].x_lin;
            s.acc_coef = co[k].x_acc;
            s.lin_lo = !last;
        };
        if (!last) {
            typename EpiApplyBase<kSplit, kNext>::Params ep = {};
            coefs(ep.s);
            e = run_apply<kSplit, kNext>(X, B, tall, L, ws, cur, kSplit || k + 2 < steps, ep, status, st);
        } else {
            typename EpiApplyBase<kSplit, kOut>::Params ep = {};
            coefs(ep.s);
            set_target<kSplit, kOut>(ep, n, O);
            e = run_apply<kSplit, kOut>(X, B, tall, L, ws, cur, false, ep, status, st);
        }
        if (e != cudaSuccess) return e;
        cur ^= 1;
    }
    return cudaSuccess;
}

// The same in one launch.
template <int kOut>
cudaError_t run_chain(const NsLayout& L, uint8_t* ws, int n, int rows, int cols, int steps,
                      const NsChainStep* co, void* const* O, long long tiles, unsigned* status,
                      cudaStream_t st) {
    constexpr auto kern = ns_chain_kernel<kOut>;
    using S = NsSmem<128>;
    const bool tall = rows > cols;
    auto at = [&](size_t off) { return reinterpret_cast<__half*>(ws + off); };
    NsChainParams<kOut> p = {};
    const NsOperand A = {{at(L.A[0]), nullptr}, L.m, L.m, n, L.ldm, L.ms};
    const NsOperand B = {{at(L.B[0]), nullptr}, L.m, L.m, n, L.ldm, L.ms};
    bool ok = ns_map(&p.map[1][0][0], A, 0, false, 128) && ns_map(&p.map[1][0][1], A, 0, false, 64);
    p.map[1][1][0] = p.map[1][0][0];
    p.map[1][1][1] = p.map[1][0][1];
    for (int cur = 0; cur < 2; ++cur) {
        const NsOperand X = {{at(L.hi[cur]), nullptr}, cols, rows, n, L.ld, L.xs};
        ok = ok && ns_map(&p.map[0][cur][0], X, 0, tall, 128) &&
             ns_map(&p.map[0][cur][1], X, 0, tall, 64) &&
             ns_map(&p.map[2][cur][0], tall ? X : B, 0, false, 128) &&
             ns_map(&p.map[2][cur][1], tall ? B : X, 0, !tall, 64);
    }
    if (!ok) return cudaErrorInvalidValue;
    p.ap.stride = static_cast<long long>(L.xs);
    p.ap.M = rows;
    p.ap.N = cols;
    p.ap.ld = L.ld;
    set_target<false, kOut>(p.ap, n, O);
    for (int k = 0; k < steps; ++k) p.step[k] = co[k];
    p.A = at(L.A[0]);
    p.B = at(L.B[0]);
    for (int h = 0; h < 2; ++h) {
        p.hi[h] = at(L.hi[h]);
        p.lo[h] = at(L.lo[h]);
    }
    p.ms = static_cast<long long>(L.ms);
    p.m = L.m;
    p.ldm = L.ldm;
    p.steps = steps;
    p.groups = n;
    p.rows = rows;
    p.cols = cols;
    p.tall = tall;
    p.count = status + 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(static_cast<unsigned>(2 * tiles), 1, 1);
    cfg.blockDim = dim3(kNsThreads, 1, 1);
    cfg.dynamicSmemBytes = S::kBytes;
    cfg.stream = st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeCooperative;
    attr[0].val.cooperative = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    note_launch();
    const cudaError_t e = cudaLaunchKernelEx(&cfg, kern, p, status, wait_limit_ns());
    if (e != cudaSuccess) cudaGetLastError();
    return e;
}

template <bool kSplit, int kOut>
cudaError_t run_iteration(const NsLayout& L, uint8_t* ws, int n, int rows, int cols, int steps,
                          const float* coeffs, void* const* O, unsigned* status,
                          cudaStream_t st) {
    NsChainStep co[kNsMaxSteps];
    if (steps > kNsMaxSteps) return cudaErrorInvalidValue;
    ns_steps(steps, coeffs, co);
    // fp16, with a cluster for every 256 x 128 tile: one launch.  (Two 256 x 384 matrices, five
    // steps: 97 us, 107 a launch per product; two 1024 x 1024 169 and 185; with two tiles to a
    // cluster, one 2048 x 2048 292 and 281.  fp32 products are longer and lost by it: two
    // 512 x 1024 matrices 288 and 265.)
    if constexpr (!kSplit) {
        const long long sym = n * ns_matrix_tiles(L.m, L.m, true),
                        app = n * ns_matrix_tiles(rows, cols, false), tiles = sym > app ? sym : app;
        constexpr auto kern = ns_chain_kernel<kOut>;
        const cudaError_t e = set_smem_limit<kern>(NsSmem<128>::kBytes);
        if (e != cudaSuccess) return e;
        DevInfo di;
        if (!current_device_info(&di)) return cudaErrorUnknown;
        if (tiles <= resident_clusters<kern>(kNsThreads, NsSmem<128>::kBytes, di.sm_count))
            return run_chain<kOut>(L, ws, n, rows, cols, steps, co, O, tiles, status, st);
    }
    return run_steps<kSplit, kOut>(L, ws, n, rows, cols, steps, co, O, status, st);
}

// G_l = g[l]^T A[l] (bf16) with the momentum in the epilogue; *parts: the partial sums per layer.
cudaError_t run_momentum(int n, int T, int rows, int cols, const NsMomentum& mom, float* U,
                         size_t u_stride, double* part, int* parts, unsigned* status,
                         cudaStream_t st) {
    EpiMomentumBase::Params ep = {};
    for (int l = 0; l < kMaxGroups; ++l) ep.M[l] = mom.M[l < n ? l : 0];
    ep.U = U;
    ep.u_stride = static_cast<long long>(u_stride);
    ep.part = part;
    ep.rows = rows;
    ep.cols = cols;
    ep.mu = mom.mu;
    ep.nesterov = mom.nesterov;
    ep.m_blocks = (rows + 255) / 256;
    DevInfo di;
    if (!current_device_info(&di)) return cudaErrorUnknown;
    const long long tiles = static_cast<long long>(n) * ep.m_blocks * ((cols + 255) / 256);
    const bool narrow = 4 * tiles <= di.sm_count;  // as in run_ns
    ep.n_blocks = narrow ? (cols + 127) / 128 : (cols + 255) / 256;
    *parts = ep.m_blocks * ep.n_blocks * 2 * kNsWarps;
    NsGradMaps maps;
    for (int l = 0; l < kMaxGroups; ++l) {
        if (l >= n) {
            maps.a[l] = maps.a[0];
            maps.b[l] = maps.b[0];
            continue;
        }
        const NsOperand g = {{static_cast<const __half*>(mom.g[l]), nullptr}, rows, T, 1, rows,
                             static_cast<size_t>(T) * rows};
        const NsOperand A = {{static_cast<const __half*>(mom.A[l]), nullptr}, cols, T, 1, cols,
                             static_cast<size_t>(T) * cols};
        if (!ns_map(&maps.a[l], g, 0, true, 64, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16) ||
            !ns_map(&maps.b[l], A, 0, true, 64, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16))
            return cudaErrorInvalidValue;
    }
    if (narrow)
        return launch_ns<128, true, true, false, EpiMomentum<128>>(maps, ep, rows, cols, T, n, false, {},
                                                                   status, st);
    return launch_ns<256, true, true, false, EpiMomentum<256>>(maps, ep, rows, cols, T, n, false, {},
                                                               status, st);
}

}  // namespace

void ns_bounds(int steps, const float* coeffs, double* bounds) {
    double u = 1.0;
    for (int k = 0; k < steps; ++k)
        bounds[k] = u = odd_max(coeffs[3 * k], coeffs[3 * k + 1], coeffs[3 * k + 2], u);
}

bool ns_coeffs_ok(int steps, const float* coeffs) {
    double u = 1.0;
    for (int k = 0; k < steps; ++k) {
        const double a = coeffs[3 * k], b = coeffs[3 * k + 1], c = coeffs[3 * k + 2];
        if (!isfinite(a) || !isfinite(b) || !isfinite(c)) return false;
        u = odd_max(a, b, c, u);
        // bounds within 2^+-16: every coefficient of an epilogue is then a normal fp32 number
        if (!(u >= 0x1p-16 && u <= 0x1p16)) return false;
        if (fabs(a) > 0x1p16 || fabs(b) > 0x1p16 || fabs(c) > 0x1p16) return false;
    }
    return true;
}

size_t ns_workspace_bytes(int n, int rows, int cols, int dtype, bool muon) {
    return ns_layout(n, rows, cols, dtype, muon).total;
}

size_t ns_clear_bytes(int n, int rows, int cols, int dtype, bool muon) {
    return ns_layout(n, rows, cols, dtype, muon).clear;
}

float* ns_update_buffer(void* ws, int n, int rows, int cols, int dtype, int layer) {
    const NsLayout L = ns_layout(n, rows, cols, dtype, true);
    return reinterpret_cast<float*>(static_cast<uint8_t*>(ws) + L.U) + layer * L.u_stride;
}

cudaError_t launch_newton_schulz(int n, int rows, int cols, int dtype, const void* const* G,
                                 const NsMomentum* mom, float eps, int steps, const float* coeffs,
                                 const NsTarget& to, void* workspace, unsigned* status,
                                 cudaStream_t st) {
    const bool split = ns_split(dtype, rows, cols), f32 = dtype == 0;
    const NsLayout L = ns_layout(n, rows, cols, dtype, mom != nullptr);
    uint8_t* ws = static_cast<uint8_t*>(workspace);
    double* part = reinterpret_cast<double*>(ws + L.part);
    const size_t numel = static_cast<size_t>(rows) * cols;
    int blocks = norm_blocks(numel);
    NsPtrs p = {};
    for (int l = 0; l < n; ++l) {
        p.in[l] = mom ? reinterpret_cast<float*>(ws + L.U) + l * L.u_stride : G[l];
        p.M[l] = mom ? mom->M[l] : nullptr;
    }
    const dim3 grid(blocks, n);
    cudaError_t e;
    if (mom && mom->g) {  // bf16, T > 0
        e = run_momentum(n, mom->T, rows, cols, *mom, reinterpret_cast<float*>(ws + L.U), L.u_stride,
                         part, &blocks, status, st);
    } else if (mom) {
        ns_momentum_kernel<<<grid, kPassThreads, 0, st>>>(p, numel, mom->mu, mom->nesterov, part),
            note_launch();
        e = cudaGetLastError();
    } else if (f32) {
        e = launch_chained(ns_norm_kernel<float>, grid, kPassThreads, 0, st, p, numel, part);
    } else {
        e = launch_chained(ns_norm_kernel<__nv_bfloat16>, grid, kPassThreads, 0, st, p, numel, part);
    }
    if (e != cudaSuccess) return e;
    if (blocks > kNormBlocks) {  // too many for every block of the cast to add up
        double* sum = reinterpret_cast<double*>(ws + L.sum);
        e = launch_chained(ns_sum_kernel, dim3(n), kSumThreads, 0, st,
                           static_cast<const double*>(part), blocks, sum);
        if (e != cudaSuccess) return e;
        part = sum;
        blocks = 1;
    }
    const size_t vecs = static_cast<size_t>(rows) * ((cols + 7) / 8);
    const size_t want = (vecs + kPassThreads - 1) / kPassThreads;
    const dim3 cgrid(static_cast<unsigned>(want < 1024 ? want : 1024), n);
    __half* hi = reinterpret_cast<__half*>(ws + L.hi[0]);
    __half* lo = reinterpret_cast<__half*>(ws + L.lo[0]);
    float* x32 = split ? reinterpret_cast<float*>(ws + L.x32) : nullptr;
    const float scale = ldexpf(1.f, scale_exp(1.0));
    auto cast = [&](auto kern) {
        return launch_chained(kern, cgrid, kPassThreads, 0, st, p, rows, cols, L.ld, part, blocks, eps,
                              scale, hi, lo, x32, L.xs);
    };
    if (f32 || mom)
        e = split ? cast(ns_cast_kernel<float, true>) : cast(ns_cast_kernel<float, false>);
    else
        e = split ? cast(ns_cast_kernel<__nv_bfloat16, true>) : cast(ns_cast_kernel<__nv_bfloat16, false>);
    if (e != cudaSuccess) return e;
    void* O32[kMaxGroups];
    if (mom)  // in place of U, which is in X_0 by now
        for (int l = 0; l < n; ++l) O32[l] = const_cast<void*>(p.in[l]);
    void* const* O = mom ? O32 : to.out;
    auto iterate = [&](auto run) { return run(L, ws, n, rows, cols, steps, coeffs, O, status, st); };
    if (f32 || mom)
        e = split ? iterate(run_iteration<true, kResult32>) : iterate(run_iteration<false, kResult32>);
    else
        e = split ? iterate(run_iteration<true, kResult>) : iterate(run_iteration<false, kResult>);
    if (e != cudaSuccess || !mom) return e;
    NsWeights w = {};
    for (int l = 0; l < n; ++l) {
        w.O[l] = static_cast<const float*>(p.in[l]);
        w.W[l] = to.W[l];
        w.out[l] = to.out ? to.out[l] : nullptr;
    }
    const size_t units = (numel + kPassThreads * 16 - 1) / (kPassThreads * 16);
    const dim3 wgrid(static_cast<unsigned>(units < 2048 ? units : 2048), n);
    if (f32)
        return launch_chained(ns_weight_kernel<float>, wgrid, kPassThreads, 0, st, w, numel, to.keep,
                              to.rate, static_cast<const unsigned*>(status));
    return launch_chained(ns_weight_kernel<__nv_bfloat16>, wgrid, kPassThreads, 0, st, w, numel,
                          to.keep, to.rate, static_cast<const unsigned*>(status));
}

}  // namespace fpo
