// adamw.cu -- one AdamW step over many tensors (Sec. 3.1's optimizer beyond the target
// matrices: biases, norm weights, any matrix with a given gradient), the moments in fp32 or in
// 8 bits, with the relative clip of App. A per tensor.
//
// A tensor is cut into chunks of 2048 elements, 8 per thread of a block; the blocks walk the
// chunks of all tensors, and a chunk's tensor is found from the table of first chunks in the
// launch's parameters.  Without a clip that is one launch.  With one, a first pass leaves
// (||W||^2, ||x||^2) of every chunk, x the step or the gradient, a second adds them per tensor
// in a fixed order, and the third takes the step scaled.
//
// 8-bit moments: 256 consecutive elements (a warp's share of a chunk) have one scale per
// moment, a power of two that brings the largest magnitude to the top of the format's range:
//   m   sign, 4 exponent bits, 3 mantissa bits (e4m3): largest |m| / scale in [2^7, 2^8)
//   v   5 exponent bits, 3 mantissa bits, no sign: largest v / scale in [2^14, 2^15)
// A code is what is left of an fp32 number's bits under its sign, shifted down by 20, once the
// number is scaled to where fp32's subnormal numbers are the format's: 2^-120 (exponent bias
// 127 to 7) and 2^-111 (to 16).
// Rounding is stochastic: 16 random bits are added below the kept ones before the rest is cut
// off, so that the expected value is the value (in steps of 2^-16 of a unit).  With beta2 0.999
// v moves by 0.1% a step and a unit is 6-12%: rounded to nearest, v would never fall, and hardly
// rise.  The bits come from a hash of the call's seed, the step, the tensor's index, the block
// and the element: the same call gives the same bits.  v > 0 is never kept as 0, where the next
// step could divide a kept m by eps alone.
// A block with a NaN or an infinity among its new m (v) gets a NaN scale: NaN throughout.
//
// Bound: HBM.
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <math.h>

#include "internal.h"

namespace fpo {
namespace {

constexpr int kThreads = 256;
constexpr int kPer = 8;                        // elements per thread
constexpr int kChunk = kThreads * kPer;        // elements of a block's turn
static_assert(kAdamBlock == 32 * kPer, "a warp's share has one scale");

// Odd words for the rounding bits: fractions of the golden ratio, sqrt(2) and sqrt(3).
constexpr uint32_t kPhi = 0x9E3779B9u, kSqrt2 = 0x6A09E667u, kSqrt3 = 0xBB67AE85u;

__host__ __device__ __forceinline__ uint32_t mix(uint32_t h) {
    h = (h ^ (h >> 16)) * kSqrt2;
    h = (h ^ (h >> 13)) * kSqrt3;
    return h ^ (h >> 16);
}

// The tensors of one launch.  Flags: g and W_out in bf16, moments in 8 bits.
enum : uint8_t { kG16 = 1, kOut16 = 2, kState8 = 4 };
template <int CAP>
struct Table {
    const void* g[CAP];
    float* w[CAP];
    void* wo[CAP];
    void* m[CAP];
    void* v[CAP];
    float* ms[CAP];
    float* vs[CAP];
    long long n[CAP];
    int first[CAP + 1];  // first chunk of each tensor; [count] is the total
    uint32_t key[CAP];
    float wd[CAP];
    uint8_t flags[CAP];
    int count;
};

__device__ __forceinline__ float2 unpack_bf16x2(uint32_t x) {
    return make_float2(__uint_as_float(x << 16), __uint_as_float(x & 0xffff0000u));
}
__device__ __forceinline__ uint32_t pack_bf16x2(float lo, float hi) {
    const __nv_bfloat162 p = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&p);
}

// 8 elements from i (a multiple of 8) of an array, those from n on as zeros.
__device__ __forceinline__ void load8(const float* p, long long i, long long n, float (&x)[kPer]) {
    if (i + kPer <= n) {
        const float4 a = *reinterpret_cast<const float4*>(p + i);
        const float4 b = *reinterpret_cast<const float4*>(p + i + 4);
        x[0] = a.x; x[1] = a.y; x[2] = a.z; x[3] = a.w;
        x[4] = b.x; x[5] = b.y; x[6] = b.z; x[7] = b.w;
    } else {
#pragma unroll
        for (int k = 0; k < kPer; ++k) x[k] = i + k < n ? p[i + k] : 0.f;
    }
}
__device__ __forceinline__ void load8(const __nv_bfloat16* p, long long i, long long n,
                                      float (&x)[kPer]) {
    if (i + kPer <= n) {
        const uint4 u = *reinterpret_cast<const uint4*>(p + i);
        const float2 a = unpack_bf16x2(u.x), b = unpack_bf16x2(u.y), c = unpack_bf16x2(u.z),
                     d = unpack_bf16x2(u.w);
        x[0] = a.x; x[1] = a.y; x[2] = b.x; x[3] = b.y;
        x[4] = c.x; x[5] = c.y; x[6] = d.x; x[7] = d.y;
    } else {
#pragma unroll
        for (int k = 0; k < kPer; ++k) x[k] = i + k < n ? __bfloat162float(p[i + k]) : 0.f;
    }
}
__device__ __forceinline__ void store8(float* p, long long i, long long n, const float (&x)[kPer]) {
    if (i + kPer <= n) {
        *reinterpret_cast<float4*>(p + i) = make_float4(x[0], x[1], x[2], x[3]);
        *reinterpret_cast<float4*>(p + i + 4) = make_float4(x[4], x[5], x[6], x[7]);
    } else {
#pragma unroll
        for (int k = 0; k < kPer; ++k)
            if (i + k < n) p[i + k] = x[k];
    }
}
__device__ __forceinline__ void store8(__nv_bfloat16* p, long long i, long long n,
                                       const float (&x)[kPer]) {
    if (i + kPer <= n) {
        *reinterpret_cast<uint4*>(p + i) =
            make_uint4(pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3]), pack_bf16x2(x[4], x[5]),
                       pack_bf16x2(x[6], x[7]));
    } else {
#pragma unroll
        for (int k = 0; k < kPer; ++k)
            if (i + k < n) p[i + k] = __float2bfloat16_rn(x[k]);
    }
}
__device__ __forceinline__ uint2 load_codes(const uint8_t* p, long long i, long long n) {
    if (i + kPer <= n) return *reinterpret_cast<const uint2*>(p + i);
    uint32_t w[2] = {0u, 0u};
#pragma unroll
    for (int k = 0; k < kPer; ++k)
        if (i + k < n) w[k / 4] |= static_cast<uint32_t>(p[i + k]) << (8 * (k % 4));
    return make_uint2(w[0], w[1]);
}
__device__ __forceinline__ void store_codes(uint8_t* p, long long i, long long n, uint2 c) {
    if (i + kPer <= n) {
        *reinterpret_cast<uint2*>(p + i) = c;
        return;
    }
    const uint32_t w[2] = {c.x, c.y};
#pragma unroll
    for (int k = 0; k < kPer; ++k)
        if (i + k < n) p[i + k] = static_cast<uint8_t>(w[k / 4] >> (8 * (k % 4)));
}

// The two formats: exponent at the block's maximum, factor to fp32's subnormal range and back.
template <bool kSigned>
struct Format {
    static constexpr int kTop = kSigned ? 7 : 14;
    static constexpr uint32_t kDown = (127u - (kSigned ? 120u : 111u)) << 23;  // 2^-120, 2^-111
    static constexpr uint32_t kUp = (127u + (kSigned ? 120u : 111u)) << 23;

    static __device__ __forceinline__ float value(uint32_t code, float scale) {
        const uint32_t mag = kSigned ? (code & 0x7fu) << 20 : code << 20;
        const float x = __uint_as_float(mag) * __uint_as_float(kUp) * scale;
        return kSigned ? __uint_as_float(__float_as_uint(x) | ((code & 0x80u) << 24)) : x;
    }
    // The scale of a block from the bits of its largest magnitude, at least 2^-100 (of a block
    // of zeros too); NaN where that is an infinity or a NaN.
    static __device__ __forceinline__ float scale(uint32_t amax) {
        const uint32_t e = amax >> 23;
        if (e == 255u) return __uint_as_float(0x7fffffffu);
        return __uint_as_float(((e > 27u ? e : 27u) - kTop) << 23);
    }
    static __device__ __forceinline__ uint32_t code(float x, float inv_scale, uint32_t u16) {
        const float y = fabsf(x) * inv_scale * __uint_as_float(kDown);
        uint32_t c = ((__float_as_uint(y) + (u16 << 4)) >> 20) & 0xffu;
        if (kSigned) return c | ((__float_as_uint(x) >> 24) & 0x80u);
        return x > 0.f && c == 0u ? 1u : c;
    }
};

template <bool kSigned>
__device__ __forceinline__ void from_codes(uint2 c, float scale, float (&x)[kPer]) {
#pragma unroll
    for (int k = 0; k < kPer; ++k)
        x[k] = Format<kSigned>::value(((k < 4 ? c.x : c.y) >> (8 * (k % 4))) & 0xffu, scale);
}

// Codes of a warp's 256 values; returns the block's scale.  r: 32 random bits per element, m
// takes the upper half and v the lower.
template <bool kSigned>
__device__ __forceinline__ float to_codes(const float (&x)[kPer], const uint32_t (&r)[kPer],
                                          uint2& c) {
    uint32_t amax = 0u;
#pragma unroll
    for (int k = 0; k < kPer; ++k) amax = max(amax, __float_as_uint(x[k]) & 0x7fffffffu);
    amax = __reduce_max_sync(0xffffffffu, amax);
    const float scale = Format<kSigned>::scale(amax);
    // of a power of two, exact
    const float inv = __uint_as_float((254u << 23) - __float_as_uint(scale));
    uint32_t w[2] = {0u, 0u};
#pragma unroll
    for (int k = 0; k < kPer; ++k) {
        const uint32_t u = kSigned ? r[k] >> 16 : r[k] & 0xffffu;
        w[k / 4] |= Format<kSigned>::code(x[k], inv, u) << (8 * (k % 4));
    }
    c = make_uint2(w[0], w[1]);
    return scale;
}

// New moments and the unclipped step of one element.  The moments' products and sums are rounded
// one by one (no FMA): an 8-bit code next to a border would otherwise depend on how the compiler
// joins them.
__device__ __forceinline__ float adamw_step(const AdamRates& op, float wd, float g, float w,
                                            float& m, float& v) {
    m = __fadd_rn(__fmul_rn(op.b1, m), __fmul_rn(op.a1, g));
    v = __fadd_rn(__fmul_rn(op.b2, v), __fmul_rn(__fmul_rn(op.a2, g), g));
    const float denom = sqrtf(v) * op.inv_sqrt_bc2 + op.eps;
    return -op.lr * (m * op.inv_bc1 / denom + wd * w);
}

// What a pass does with a chunk: the clip's sums (kNorms, of the step where op.clip is 1, else
// of the gradient) or the step itself.
template <bool kNorms, bool kState8>
__device__ __forceinline__ void chunk(const AdamRates& op, float wd, uint32_t key, bool g16,
                                      bool out16, const void* g_, float* w_, void* wo_, void* m_,
                                      void* v_, float* ms_, float* vs_, long long i, long long n,
                                      float gscale, float sscale, float& ww, float& xx) {
    float g[kPer], w[kPer], m[kPer], v[kPer];
    const long long block = i / kAdamBlock;
    const bool any = block * kAdamBlock < n;  // of the warp's 256 elements
    if (g16)
        load8(static_cast<const __nv_bfloat16*>(g_), i, n, g);
    else
        load8(static_cast<const float*>(g_), i, n, g);
    load8(w_, i, n, w);
    if (kNorms && op.clip == 2) {  // the gradient's norm needs no state
#pragma unroll
        for (int k = 0; k < kPer; ++k) {
            ww = fmaf(w[k], w[k], ww);
            xx = fmaf(g[k], g[k], xx);
        }
        return;
    }
    if constexpr (kState8) {
        const uint2 mc = load_codes(static_cast<const uint8_t*>(m_), i, n);
        const uint2 vc = load_codes(static_cast<const uint8_t*>(v_), i, n);
        from_codes<true>(mc, any ? ms_[block] : 0.f, m);
        from_codes<false>(vc, any ? vs_[block] : 0.f, v);
    } else {
        load8(static_cast<const float*>(m_), i, n, m);
        load8(static_cast<const float*>(v_), i, n, v);
    }
#pragma unroll
    for (int k = 0; k < kPer; ++k) {
        const float st = adamw_step(op, wd, gscale * g[k], w[k], m[k], v[k]);
        if constexpr (kNorms) {
            const float d = i + k < n ? st : 0.f;
            ww = fmaf(w[k], w[k], ww);
            xx = fmaf(d, d, xx);
        } else {
            w[k] = fmaf(sscale, st, w[k]);
        }
    }
    if constexpr (!kNorms) {
        store8(w_, i, n, w);
        if (wo_) {
            if (out16)
                store8(static_cast<__nv_bfloat16*>(wo_), i, n, w);
            else
                store8(static_cast<float*>(wo_), i, n, w);
        }
        if constexpr (kState8) {
            const uint32_t lane = threadIdx.x & 31u;
            uint32_t h = mix(key ^ static_cast<uint32_t>(block)) + lane * kPer * kPhi;
            uint32_t r[kPer];
#pragma unroll
            for (int k = 0; k < kPer; ++k, h += kPhi) {
                r[k] = (h ^ (h >> 15)) * kSqrt2;
                r[k] ^= r[k] >> 16;
            }
            uint2 mc, vc;
            const float msc = to_codes<true>(m, r, mc);
            const float vsc = to_codes<false>(v, r, vc);
            if (!any) return;
            store_codes(static_cast<uint8_t*>(m_), i, n, mc);
            store_codes(static_cast<uint8_t*>(v_), i, n, vc);
            if (lane == 0) {
                ms_[block] = msc;
                vs_[block] = vsc;
            }
        } else {
            store8(static_cast<float*>(m_), i, n, m);
            store8(static_cast<float*>(v_), i, n, v);
        }
    }
}

__device__ __forceinline__ float warp_sum(float x) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
    return x;
}

// kNorms: part[chunk] = the chunk's two sums.  Else scales[tensor] (null: 1) clips the step.
template <int CAP, bool kNorms>
__global__ void __launch_bounds__(kThreads)
    adamw_kernel(const __grid_constant__ Table<CAP> t, const __grid_constant__ AdamRates op,
                 float2* __restrict__ part, const float* __restrict__ scales) {
    const int total = t.first[t.count];
    int k = 0;
    for (int c = blockIdx.x; c < total; c += gridDim.x) {
        // the chunk's tensor: the last whose first chunk is not behind it (some have none)
        int hi = t.count;
        while (hi - k > 1) {
            const int mid = (k + hi) / 2;
            if (t.first[mid] <= c)
                k = mid;
            else
                hi = mid;
        }
        const long long i = static_cast<long long>(c - t.first[k]) * kChunk + threadIdx.x * kPer;
        const uint8_t f = t.flags[k];
        const float sc = scales ? scales[k] : 1.f;
        const float gscale = op.clip == 2 ? sc : 1.f, sscale = op.clip == 1 ? sc : 1.f;
        float ww = 0.f, xx = 0.f;
        if (f & kState8)
            chunk<kNorms, true>(op, t.wd[k], t.key[k], f & kG16, f & kOut16, t.g[k], t.w[k], t.wo[k],
                                t.m[k], t.v[k], t.ms[k], t.vs[k], i, t.n[k], gscale, sscale, ww, xx);
        else
            chunk<kNorms, false>(op, t.wd[k], t.key[k], f & kG16, f & kOut16, t.g[k], t.w[k],
                                 t.wo[k], t.m[k], t.v[k], t.ms[k], t.vs[k], i, t.n[k], gscale,
                                 sscale, ww, xx);
        if constexpr (kNorms) {
            __shared__ float2 sh[kThreads / 32];
            ww = warp_sum(ww);
            xx = warp_sum(xx);
            __syncthreads();  // the chunk before is read
            if ((threadIdx.x & 31) == 0) sh[threadIdx.x / 32] = make_float2(ww, xx);
            __syncthreads();
            if (threadIdx.x == 0) {
                float2 s = sh[0];
                for (int q = 1; q < kThreads / 32; ++q) {
                    s.x += sh[q].x;
                    s.y += sh[q].y;
                }
                part[c] = s;
            }
        }
    }
}

// scales[k] = min(1, clip_frac ||W|| / ||x||) from the tensor's chunk sums: thread-strided
// fp64, a fixed butterfly, then the warps in order.
template <int CAP>
__global__ void __launch_bounds__(kThreads)
    adamw_scale_kernel(const __grid_constant__ Table<CAP> t, const float2* __restrict__ part,
                       float clip_frac, float* __restrict__ scales) {
    const int k = blockIdx.x;
    double ww = 0.0, xx = 0.0;
    for (int c = t.first[k] + threadIdx.x; c < t.first[k + 1]; c += kThreads) {
        ww += part[c].x;
        xx += part[c].y;
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
        ww += __shfl_xor_sync(0xffffffffu, ww, o);
        xx += __shfl_xor_sync(0xffffffffu, xx, o);
    }
    __shared__ double sh[2][kThreads / 32];
    if ((threadIdx.x & 31) == 0) {
        sh[0][threadIdx.x / 32] = ww;
        sh[1][threadIdx.x / 32] = xx;
    }
    __syncthreads();
    if (threadIdx.x != 0) return;
    ww = xx = 0.0;
    for (int q = 0; q < kThreads / 32; ++q) {
        ww += sh[0][q];
        xx += sh[1][q];
    }
    const double lim = static_cast<double>(clip_frac) * sqrt(ww);
    scales[k] = static_cast<float>(sqrt(xx) > lim ? lim / sqrt(xx) : 1.0);
}

// out[i] = the value of an 8-bit moment (exact in bf16: 4 significant bits times a power of two).
template <bool kSigned, typename Out>
__global__ void __launch_bounds__(kThreads)
    state_values_kernel(const uint8_t* __restrict__ codes, const float* __restrict__ scales,
                        long long n, Out* __restrict__ out) {
    const long long i = (blockIdx.x * static_cast<long long>(kThreads) + threadIdx.x) * kPer;
    if (i >= n) return;
    float x[kPer];
    from_codes<kSigned>(load_codes(codes, i, n), scales[i / kAdamBlock], x);
    store8(out, i, n, x);
}

long long chunks_of(long long n) { return (n + kChunk - 1) / kChunk; }

template <int CAP>
cudaError_t run_adamw(int first, int count, const AdamTensor* ts, const AdamRates& op,
                      uint32_t key, float2* part, float* scales, cudaStream_t st) {
    Table<CAP> t = {};
    long long total = 0;
    for (int k = 0; k < count; ++k) {
        const AdamTensor& a = ts[first + k];
        t.g[k] = a.G;
        t.w[k] = a.W;
        t.wo[k] = a.W_out;
        t.m[k] = a.m;
        t.v[k] = a.v;
        t.ms[k] = a.m_scale;
        t.vs[k] = a.v_scale;
        t.n[k] = a.n;
        t.first[k] = static_cast<int>(total);
        t.key[k] = mix(key + static_cast<uint32_t>(first + k));
        t.wd[k] = a.weight_decay;
        t.flags[k] = static_cast<uint8_t>((a.g_bf16 ? kG16 : 0) | (a.out_bf16 ? kOut16 : 0) |
                                          (a.state8 ? kState8 : 0));
        total += chunks_of(a.n);
    }
    t.count = count;
    t.first[count] = static_cast<int>(total);
    if (total == 0) return cudaSuccess;
    if (total > 0x7fffffff) return cudaErrorInvalidValue;
    DevInfo di;
    if (!current_device_info(&di)) return cudaErrorUnknown;
    const long long most = 8LL * di.sm_count;
    const unsigned grid = static_cast<unsigned>(total < most ? total : most);
    if (op.clip != 0) {
        adamw_kernel<CAP, true><<<grid, kThreads, 0, st>>>(t, op, part, nullptr), note_launch();
        cudaError_t e = cudaGetLastError();
        if (e != cudaSuccess) return e;
        adamw_scale_kernel<CAP><<<count, kThreads, 0, st>>>(t, part, op.clip_frac, scales),
            note_launch();
        e = cudaGetLastError();
        if (e != cudaSuccess) return e;
    }
    adamw_kernel<CAP, false><<<grid, kThreads, 0, st>>>(t, op, nullptr,
                                                         op.clip != 0 ? scales : nullptr),
        note_launch();
    return cudaGetLastError();
}

}  // namespace

// Tensors of one launch: the table of a few is a tenth of the parameters of many.
constexpr int kFew = 12, kMany = 128;

size_t adamw_workspace_floats(int n_tensors, const int64_t* n) {
    long long most = 0;
    for (int f = 0; f < n_tensors; f += kMany) {
        long long total = 0;
        for (int k = f; k < n_tensors && k < f + kMany; ++k) total += chunks_of(n[k]);
        most = total > most ? total : most;
    }
    return static_cast<size_t>(kMany + 2 * most);  // the scales, then the chunks' sums
}

cudaError_t launch_adamw(int n_tensors, const AdamTensor* ts, const AdamRates& op, uint64_t seed,
                         int64_t step, float* ws, cudaStream_t st) {
    uint32_t key = mix(static_cast<uint32_t>(seed) + kPhi);
    key = mix(key ^ static_cast<uint32_t>(seed >> 32));
    key = mix(key ^ static_cast<uint32_t>(step));
    float2* part = reinterpret_cast<float2*>(ws ? ws + kMany : nullptr);
    for (int f = 0; f < n_tensors; f += kMany) {
        const int count = n_tensors - f < kMany ? n_tensors - f : kMany;
        const cudaError_t e = count <= kFew ? run_adamw<kFew>(f, count, ts, op, key, part, ws, st)
                                            : run_adamw<kMany>(f, count, ts, op, key, part, ws, st);
        if (e != cudaSuccess) return e;
    }
    return cudaSuccess;
}

cudaError_t launch_state_values(bool is_signed, long long n, const void* codes, const float* scales,
                                int out_dtype, void* out, cudaStream_t st) {
    const long long blocks = (n + kChunk - 1) / kChunk;
    if (blocks > 0x7fffffff) return cudaErrorInvalidValue;
    const unsigned grid = static_cast<unsigned>(blocks);
    const uint8_t* c = static_cast<const uint8_t*>(codes);
    if (is_signed) {
        if (out_dtype == 1)
            state_values_kernel<true><<<grid, kThreads, 0, st>>>(c, scales, n, static_cast<__nv_bfloat16*>(out));
        else
            state_values_kernel<true><<<grid, kThreads, 0, st>>>(c, scales, n, static_cast<float*>(out));
    } else {
        if (out_dtype == 1)
            state_values_kernel<false><<<grid, kThreads, 0, st>>>(c, scales, n, static_cast<__nv_bfloat16*>(out));
        else
            state_values_kernel<false><<<grid, kThreads, 0, st>>>(c, scales, n, static_cast<float*>(out));
    }
    note_launch();
    return cudaGetLastError();
}

}  // namespace fpo
