// adamw.cu -- one AdamW step over many tensors (Sec. 3.1's optimizer beyond the target
// matrices: biases, norm weights, any matrix with a given gradient), the moments in fp32 or in
// 8 bits, with the relative clip of App. A per tensor.
//
// A tensor is cut into chunks, 128 elements per warp of a block and quad of a lane (so that every
// access of a warp is whole lines): 4 quads with fp32 moments, whose traffic wants the loads in
// flight, 2 with 8-bit ones, whose arithmetic wants the warps.  A block takes one chunk of any
// tensor, found from the table of first chunks in the launch's parameters.  Blocks that stay and
// walk the chunks were slower, their warps in step with one another between loading and storing
// (90M elements, bf16 gradients, us: fp32 moments 361, resident blocks 395, with 2 quads 445; 8-bit
// ones, before their arithmetic was thinned out to the present 238, 262, 265, with 4 quads 299).
// Without a clip that is one launch.  With one, a first pass leaves (||W||^2, ||x||^2) of every
// chunk, x the step or the gradient, a second adds them per tensor in a fixed order, and the third
// takes the step scaled.
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
// Bound: HBM.  90M elements, no clip, step clip, gradient clip: fp32 moments 361 us (7.0 TB/s of the 28
// bytes an element), 515 (two passes' 516 at the copy rate), 470; 8-bit moments 237 (6.1 TB/s of 16;
// the rounding's hash and the scales' maxima take issue slots), 390, 342 (the norms pass computes the
// step a second time, for keeping it would cost more bytes than the moments).  Squares outside fp32's
// range are added a second time, scaled: gradients of zeros, which look like such, take 477 for 468.
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <math.h>

#include "internal.h"

namespace fpo {
namespace {

constexpr int kThreads = 256;
// Quads of a lane, elements of a thread, a warp and a block's turn.  Element 4 q + i of a lane is
// 128 q + 4 lane + i of its warp's.
template <bool kState8>
struct Share {
    static constexpr int kQuads = kState8 ? 2 : 4;
    static constexpr int kPer = 4 * kQuads;
    static constexpr int kWarp = 32 * kPer;
    static constexpr int kChunk = kThreads / 32 * kWarp;
};
static_assert(Share<true>::kWarp == kAdamBlock, "a warp's share has one scale");

// Odd words for the rounding bits: fractions of the golden ratio, sqrt(2) and sqrt(3).
constexpr uint32_t kPhi = 0x9E3779B9u, kSqrt2 = 0x6A09E667u, kSqrt3 = 0xBB67AE85u;

__host__ __device__ __forceinline__ uint32_t mix(uint32_t h) {
    h = (h ^ (h >> 16)) * kSqrt2;
    h = (h ^ (h >> 13)) * kSqrt3;
    return h ^ (h >> 16);
}

// The tensors of one launch.  Flags: g and W_out in bf16.
enum : uint8_t { kG16 = 1, kOut16 = 2 };
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

// Four elements from i (a multiple of 4) of an array; not kFull: those from n on are zeros, and
// stay as they are.
template <bool kFull>
__device__ __forceinline__ void load4(const float* p, long long i, long long n, float* x) {
    if (kFull || i + 4 <= n) {
        const float4 a = *reinterpret_cast<const float4*>(p + i);
        x[0] = a.x; x[1] = a.y; x[2] = a.z; x[3] = a.w;
    } else {
#pragma unroll
        for (int k = 0; k < 4; ++k) x[k] = i + k < n ? p[i + k] : 0.f;
    }
}
template <bool kFull>
__device__ __forceinline__ void load4(const __nv_bfloat16* p, long long i, long long n, float* x) {
    if (kFull || i + 4 <= n) {
        const uint2 u = *reinterpret_cast<const uint2*>(p + i);
        const float2 a = unpack_bf16x2(u.x), b = unpack_bf16x2(u.y);
        x[0] = a.x; x[1] = a.y; x[2] = b.x; x[3] = b.y;
    } else {
#pragma unroll
        for (int k = 0; k < 4; ++k) x[k] = i + k < n ? __bfloat162float(p[i + k]) : 0.f;
    }
}
template <bool kFull>
__device__ __forceinline__ void store4(float* p, long long i, long long n, const float* x) {
    if (kFull || i + 4 <= n) {
        *reinterpret_cast<float4*>(p + i) = make_float4(x[0], x[1], x[2], x[3]);
    } else {
#pragma unroll
        for (int k = 0; k < 4; ++k)
            if (i + k < n) p[i + k] = x[k];
    }
}
template <bool kFull>
__device__ __forceinline__ void store4(__nv_bfloat16* p, long long i, long long n, const float* x) {
    if (kFull || i + 4 <= n) {
        *reinterpret_cast<uint2*>(p + i) = make_uint2(pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3]));
    } else {
#pragma unroll
        for (int k = 0; k < 4; ++k)
            if (i + k < n) p[i + k] = __float2bfloat16_rn(x[k]);
    }
}
template <bool kFull>
__device__ __forceinline__ uint32_t load_codes(const uint8_t* p, long long i, long long n) {
    if (kFull || i + 4 <= n) return *reinterpret_cast<const uint32_t*>(p + i);
    uint32_t w = 0u;
#pragma unroll
    for (int k = 0; k < 4; ++k)
        if (i + k < n) w |= static_cast<uint32_t>(p[i + k]) << (8 * k);
    return w;
}
template <bool kFull>
__device__ __forceinline__ void store_codes(uint8_t* p, long long i, long long n, uint32_t c) {
    if (kFull || i + 4 <= n) {
        *reinterpret_cast<uint32_t*>(p + i) = c;
        return;
    }
#pragma unroll
    for (int k = 0; k < 4; ++k)
        if (i + k < n) p[i + k] = static_cast<uint8_t>(c >> (8 * k));
}

__device__ __forceinline__ float2 both(float x) { return make_float2(x, x); }

// The two formats: exponent at the block's maximum, factor to fp32's subnormal range and back.
template <bool kSigned>
struct Format {
    static constexpr int kTop = kSigned ? 7 : 14;
    static constexpr uint32_t kDown = (127u - (kSigned ? 120u : 111u)) << 23;  // 2^-120, 2^-111
    static constexpr uint32_t kUp = (127u + (kSigned ? 120u : 111u)) << 23;

    // The scale of a block from the bits of its largest magnitude, at least 2^-100 (of a block
    // of zeros too); NaN where that is an infinity or a NaN.
    static __device__ __forceinline__ float scale(uint32_t amax) {
        const uint32_t e = amax >> 23;
        if (e == 255u) return __uint_as_float(0x7fffffffu);
        return __uint_as_float(((e > 27u ? e : 27u) - kTop) << 23);
    }
};

// The values of four codes (m by the hardware's conversion of e4m3 to fp16, which is exact).
template <bool kSigned>
__device__ __forceinline__ void from_codes(uint32_t c, float scale, float* x) {
#pragma unroll
    for (int k = 0; k < 4; k += 2) {
        float2 v;
        if constexpr (kSigned) {
            uint32_t h;
            asm("{\n\t.reg .b16 lo, hi;\n\tmov.b32 {lo, hi}, %1;\n\tcvt.rn.f16x2.e4m3x2 %0, lo;\n\t}"
                : "=r"(h)
                : "r"(c >> (8 * k)));
            v = __half22float2(*reinterpret_cast<const __half2*>(&h));
        } else {
            const uint32_t a = k == 0 ? c << 20 : c << 4, b = k == 0 ? c << 12 : c >> 4;
            v = __fmul2_rn(make_float2(__uint_as_float(a & 0x0ff00000u), __uint_as_float(b & 0x0ff00000u)),
                           both(__uint_as_float(Format<false>::kUp)));
        }
        v = __fmul2_rn(v, both(scale));  // (2^111 and the scale apart: their product may be out of range)
        x[k] = v.x;
        x[k + 1] = v.y;
    }
}

// max(|a|, |b|), NaN where either is.
__device__ __forceinline__ float max_abs(float a, float b) {
    float m;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(m) : "f"(fabsf(a)), "f"(fabsf(b)));
    return m;
}

// Codes of a warp's block of 256 values, eight per lane (x, and 32 random bits r of each: m takes
// the upper half, v the lower); returns the block's scale.
template <bool kSigned>
__device__ __forceinline__ float to_codes(const float* x, const uint32_t* r, uint32_t (&c)[2]) {
    float top = max_abs(x[0], x[1]);
#pragma unroll
    for (int k = 2; k < 8; ++k) top = max_abs(top, x[k]);
    const float scale =
        Format<kSigned>::scale(__reduce_max_sync(0xffffffffu, __float_as_uint(top) & 0x7fffffffu));
    // of a power of two, exact
    const float inv = __uint_as_float((254u << 23) - __float_as_uint(scale));
    uint32_t code[8];
#pragma unroll
    for (int k = 0; k < 8; k += 2) {
        float2 y = __fmul2_rn(make_float2(x[k], x[k + 1]), both(inv));
        y = __fmul2_rn(y, both(__uint_as_float(Format<kSigned>::kDown)));
        const uint32_t b[2] = {__float_as_uint(y.x), __float_as_uint(y.y)};
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const uint32_t u = kSigned ? r[k + i] >> 16 : r[k + i] & 0xffffu;
            const uint32_t t = b[i] + (u << 4);  // (a sign stays: bits 27 to 30 are 0)
            if (kSigned)
                code[k + i] = (t >> 20) | ((t >> 24) & 0x80u);  // (its byte is what counts)
            else
                code[k + i] = x[k + i] > 0.f ? max(t >> 20, 1u) : t >> 20;
        }
    }
#pragma unroll
    for (int k = 0; k < 2; ++k)  // their low bytes
        c[k] = __byte_perm(__byte_perm(code[4 * k], code[4 * k + 1], 0x0040),
                           __byte_perm(code[4 * k + 2], code[4 * k + 3], 0x0040), 0x5410);
    return scale;
}

__device__ __forceinline__ float sqrt_approx(float x) {
    float y;
    asm("sqrt.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ float rcp_approx(float x) {
    float y;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// New moments and the unclipped steps of a thread's elements.  The moments' products and sums are
// rounded one by one (no FMA): an 8-bit code next to a border would otherwise depend on how the
// compiler joins them.  Square root and reciprocal are the MUFU's, within 2^-22 of the step, which
// is itself some 2^-10 of a weight.
// a + b on its own: packed products and sums are joined to FMAs, also where they are written with
// .rn (27% of the moments differed); a product with a factor of 1 that the compiler does not know is
// not.
__device__ __forceinline__ float2 add_rn(float2 a, float2 b, float one) {
    return __ffma2_rn(a, both(one), b);
}

// kNew: m and v advance by g; else they have.  d: the unclipped step.
template <bool kNew, int kPer>
__device__ __forceinline__ void adamw_step(const AdamRates& op, float wd, float gscale,
                                           const float (&g)[kPer], const float (&w)[kPer],
                                           float (&m)[kPer], float (&v)[kPer], float (&d)[kPer]) {
#pragma unroll
    for (int k = 0; k < kPer; k += 2) {
        float2 m2 = make_float2(m[k], m[k + 1]), v2 = make_float2(v[k], v[k + 1]);
        if constexpr (kNew) {
            const float2 g2 = __fmul2_rn(make_float2(g[k], g[k + 1]), both(gscale));
            m2 = add_rn(__fmul2_rn(both(op.b1), m2), __fmul2_rn(both(op.a1), g2), op.one);
            v2 = add_rn(__fmul2_rn(both(op.b2), v2), __fmul2_rn(__fmul2_rn(both(op.a2), g2), g2), op.one);
            m[k] = m2.x;
            m[k + 1] = m2.y;
            v[k] = v2.x;
            v[k + 1] = v2.y;
        }
        const float2 den = __ffma2_rn(make_float2(sqrt_approx(v2.x), sqrt_approx(v2.y)),
                                      both(op.inv_sqrt_bc2), both(op.eps));
        const float2 q = __fmul2_rn(__fmul2_rn(m2, both(op.inv_bc1)),
                                    make_float2(rcp_approx(den.x), rcp_approx(den.y)));
        const float2 s = __fmul2_rn(__ffma2_rn(both(wd), make_float2(w[k], w[k + 1]), q), both(-op.lr));
        d[k] = s.x;
        d[k + 1] = s.y;
    }
}

__device__ __forceinline__ float warp_sum(float x) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
    return x;
}

// Sums of squares as 32-bit words.  In [2^-100, 2^90] (a launch's 2^31 chunks then stay in range, and
// what squares lose under fp32's numbers is below 2^-40 of the sum), 0, an infinity or a NaN: the fp32
// number.  Else, marked by the sign bit, the upper half of a double, rounded: 2^-21 of the sum.
__device__ __forceinline__ float wide_word(double x) {
    const long long b = __double_as_longlong(x) + 0x80000000ll;
    return __uint_as_float(static_cast<uint32_t>(b >> 32) | 0x80000000u);
}
__device__ __forceinline__ bool is_wide(float word) { return __float_as_int(word) < 0; }
__device__ __forceinline__ double wide_value(float word) {
    return __hiloint2double(__float_as_int(word) & 0x7fffffff, 0);
}

__device__ __forceinline__ bool in_range(float s) { return s >= 0x1p-100f && s <= 0x1p90f; }

// The word of a warp's values whose sum of squares s is not in range: magnitudes below 2^-50, or some
// from 2^40 up to 2^128, are squared where fp32 has their squares.
template <int kPer>
__device__ __forceinline__ float far_square_sum(float s, const float (&x)[kPer]) {
    const bool low = s < 0x1p-100f;
    const float f = low ? 0x1p100f : 0x1p-70f;
    float t = 0.f;
#pragma unroll
    for (int k = 0; k < kPer; ++k) t = fmaf(x[k] * f, x[k] * f, t);
    t = warp_sum(t);
    if (t == 0.f || !(t < __int_as_float(0x7f800000))) return fabsf(t);
    return wide_word(static_cast<double>(t) * (low ? 0x1p-200 : 0x1p140));
}

// The words of a warp's weights and of its gradients or steps, the same in every lane.
template <int kPer>
__device__ __forceinline__ void square_sums(const float (&w)[kPer], const float (&x)[kPer], float& ww,
                                            float& xx) {
    ww = xx = 0.f;
#pragma unroll
    for (int k = 0; k < kPer; ++k) {
        ww = fmaf(w[k], w[k], ww);
        xx = fmaf(x[k], x[k], xx);
    }
    ww = warp_sum(ww);
    xx = warp_sum(xx);
    if (in_range(ww) && in_range(xx)) return;
    if (!in_range(ww)) ww = far_square_sum(ww, w);
    if (!in_range(xx)) xx = far_square_sum(xx, x);
}

// One tensor's entry of the table.
struct Entry {
    const void* g;
    float* w;
    void* wo;
    void* m;
    void* v;
    float* ms;
    float* vs;
    long long n;
    uint32_t key;
    float wd;
    bool g16, out16;
};

// The passes.  kStep: the whole step.  kNorms: the clip's sums, of the step where op.clip is 1, else
// of the gradient.  fp32 moments with the clip on the step advance in the first pass already
// (kMoments), and the step is taken from them (kApply): 40 bytes an element instead of 42.  (8-bit
// ones would have been rounded by then.)
enum Pass { kStep, kNorms, kMoments, kApply };

// What a pass does with a warp's elements from i0.  kFull: all of them are there; else the first at
// least is.  ww, xx: the words of a pass with sums.
template <Pass kPass, bool kState8, bool kFull>
__device__ __forceinline__ void take(const AdamRates& op, const Entry& e, long long i0, float gscale,
                                     float sscale, float& ww, float& xx) {
    constexpr int kQuads = Share<kState8>::kQuads, kPer = Share<kState8>::kPer;
    float g[kPer], w[kPer], m[kPer], v[kPer];
    const int lane = threadIdx.x & 31;
    const long long n = e.n, i1 = i0 + 4 * lane;
    if (kPass == kApply) {
        // no gradient is needed
    } else if (e.g16) {
#pragma unroll
        for (int q = 0; q < kQuads; ++q)
            load4<kFull>(static_cast<const __nv_bfloat16*>(e.g), i1 + 128 * q, n, g + 4 * q);
    } else {
#pragma unroll
        for (int q = 0; q < kQuads; ++q)
            load4<kFull>(static_cast<const float*>(e.g), i1 + 128 * q, n, g + 4 * q);
    }
#pragma unroll
    for (int q = 0; q < kQuads; ++q) load4<kFull>(e.w, i1 + 128 * q, n, w + 4 * q);
    if (kPass == kNorms && op.clip == 2) {  // the gradient's norm needs no state
        square_sums(w, g, ww, xx);
        return;
    }
    const long long block = i0 / kAdamBlock;
    if constexpr (kState8) {
        const float msc = e.ms[block], vsc = e.vs[block];
        uint32_t mc[kQuads], vc[kQuads];
#pragma unroll
        for (int q = 0; q < kQuads; ++q) {
            mc[q] = load_codes<kFull>(static_cast<const uint8_t*>(e.m), i1 + 128 * q, n);
            vc[q] = load_codes<kFull>(static_cast<const uint8_t*>(e.v), i1 + 128 * q, n);
        }
#pragma unroll
        for (int q = 0; q < kQuads; ++q) {
            from_codes<true>(mc[q], msc, m + 4 * q);
            from_codes<false>(vc[q], vsc, v + 4 * q);
        }
    } else {
#pragma unroll
        for (int q = 0; q < kQuads; ++q) {
            load4<kFull>(static_cast<const float*>(e.m), i1 + 128 * q, n, m + 4 * q);
            load4<kFull>(static_cast<const float*>(e.v), i1 + 128 * q, n, v + 4 * q);
        }
    }
    float d[kPer];
    adamw_step<kPass != kApply>(op, e.wd, gscale, g, w, m, v, d);
    auto store_moments = [&] {
#pragma unroll
        for (int q = 0; q < kQuads; ++q) {
            store4<kFull>(static_cast<float*>(e.m), i1 + 128 * q, n, m + 4 * q);
            store4<kFull>(static_cast<float*>(e.v), i1 + 128 * q, n, v + 4 * q);
        }
    };
    if constexpr (kPass == kNorms || kPass == kMoments) {
        if constexpr (!kFull) {
#pragma unroll
            for (int k = 0; k < kPer; ++k)  // (no element: eps 0 would divide by 0)
                if (i1 + 128 * (k / 4) + k % 4 >= n) d[k] = 0.f;
        }
        if constexpr (kPass == kMoments) store_moments();
        square_sums(w, d, ww, xx);
        return;
    }
#pragma unroll
    for (int k = 0; k < kPer; ++k) w[k] = fmaf(sscale, d[k], w[k]);
#pragma unroll
    for (int q = 0; q < kQuads; ++q) store4<kFull>(e.w, i1 + 128 * q, n, w + 4 * q);
    if (e.wo) {
#pragma unroll
        for (int q = 0; q < kQuads; ++q) {
            if (e.out16)
                store4<kFull>(static_cast<__nv_bfloat16*>(e.wo), i1 + 128 * q, n, w + 4 * q);
            else
                store4<kFull>(static_cast<float*>(e.wo), i1 + 128 * q, n, w + 4 * q);
        }
    }
    if constexpr (kState8) {
        const uint32_t h0 = mix(e.key ^ static_cast<uint32_t>(block)) + 4u * lane * kPhi;
        uint32_t r[kPer];
#pragma unroll
        for (int k = 0; k < kPer; ++k) {
            const uint32_t h = h0 + (128u * (k / 4) + k % 4) * kPhi;
            r[k] = (h ^ (h >> 15)) * kSqrt2;
            r[k] ^= r[k] >> 16;
        }
        uint32_t mc[kQuads], vc[kQuads];
        const float msc = to_codes<true>(m, r, mc);
        const float vsc = to_codes<false>(v, r, vc);
#pragma unroll
        for (int q = 0; q < kQuads; ++q) {
            store_codes<kFull>(static_cast<uint8_t*>(e.m), i1 + 128 * q, n, mc[q]);
            store_codes<kFull>(static_cast<uint8_t*>(e.v), i1 + 128 * q, n, vc[q]);
        }
        if (lane == 0) {
            e.ms[block] = msc;
            e.vs[block] = vsc;
        }
    } else if constexpr (kPass == kStep) {
        store_moments();
    }
}

// The word of the block's, from its warps' in order.
__device__ __forceinline__ float add_words(const float* words) {
    float s = words[0];
    bool wide = is_wide(s);
    for (int i = 1; i < kThreads / 32; ++i) {
        s += words[i];
        wide |= is_wide(words[i]);
    }
    if (!wide) return fabsf(s);  // (a NaN's sign bit is no mark)
    double d = 0.0;
    for (int i = 0; i < kThreads / 32; ++i)
        d += is_wide(words[i]) ? wide_value(words[i]) : static_cast<double>(words[i]);
    if (d < 0x1p-100 || (d > 0x1p90 && isfinite(d))) return wide_word(d);
    return fabsf(static_cast<float>(d));
}

constexpr bool sums(Pass p) { return p == kNorms || p == kMoments; }

// Passes with sums: part[chunk] = the words of the chunk's two.  Else scales[tensor] (null: 1) clips the step.
template <int CAP, Pass kPass, bool kState8>
__global__ void __launch_bounds__(kThreads, kPass == kNorms ? (kState8 ? 5 : 3) : (kState8 ? 4 : 2))
    adamw_kernel(const __grid_constant__ Table<CAP> t, const __grid_constant__ AdamRates op,
                 float2* __restrict__ part, const float* __restrict__ scales) {
    using S = Share<kState8>;
    const int warp = threadIdx.x / 32;
    // behind a norms pass from the end: what that pass read last is still in L2
    const int c = !sums(kPass) && scales ? gridDim.x - 1 - blockIdx.x : blockIdx.x;
    int k = 0, hi = t.count;  // the chunk's tensor: the last whose first chunk is not behind it
    while (hi - k > 1) {
        const int mid = (k + hi) / 2;
        if (t.first[mid] <= c)
            k = mid;
        else
            hi = mid;
    }
    const Entry e{t.g[k],  t.w[k], t.wo[k],  t.m[k],  t.v[k], t.ms[k],
                  t.vs[k], t.n[k], t.key[k], t.wd[k], (t.flags[k] & kG16) != 0,
                  (t.flags[k] & kOut16) != 0};
    const long long i0 = static_cast<long long>(c - t.first[k]) * S::kChunk + warp * S::kWarp;
    const float sc = scales ? scales[k] : 1.f;
    const float gscale = op.clip == 2 ? sc : 1.f, sscale = op.clip == 1 ? sc : 1.f;
    float ww = 0.f, xx = 0.f;
    if (i0 + S::kWarp <= e.n)
        take<kPass, kState8, true>(op, e, i0, gscale, sscale, ww, xx);
    else if (i0 < e.n)
        take<kPass, kState8, false>(op, e, i0, gscale, sscale, ww, xx);
    if constexpr (sums(kPass)) {
        __shared__ float sh[2][kThreads / 32];
        if ((threadIdx.x & 31) == 0) {
            sh[0][warp] = ww;
            sh[1][warp] = xx;
        }
        __syncthreads();
        if (warp < 2 && (threadIdx.x & 31) == 0) reinterpret_cast<float*>(part + c)[warp] = add_words(sh[warp]);
    }
}

// A sum of words: of the fp32 numbers with what the additions rounded off (Knuth's two-sum), 48 bits in
// all, and of the wide ones in fp64.
struct TwoSum {
    float hi = 0.f, lo = 0.f;
    double wide = 0.0;
    __device__ __forceinline__ void add(float x) {
        const float s = __fadd_rn(hi, x), b = __fsub_rn(s, hi);
        lo = __fadd_rn(lo, __fadd_rn(__fsub_rn(hi, __fsub_rn(s, b)), __fsub_rn(x, b)));
        hi = s;
    }
    __device__ __forceinline__ void add_word(float x) {
        if (is_wide(x))
            wide += wide_value(x);
        else
            add(x);
    }
    __device__ __forceinline__ double value() const {
        return isfinite(hi) ? static_cast<double>(hi) + lo + wide : static_cast<double>(hi);
    }
};

// scales[k] = min(1, clip_frac ||W|| / ||x||) from the tensor's chunk sums (words): thread-strided, a fixed
// butterfly, then the warps in order.  One block per tensor, whose few fp64 adders would take 10 us
// for the 22,000 chunks of 45M elements (20 to 33 us with loads one by one); the threads add pairs
// of fp32 numbers instead, eight loads ahead.
constexpr int kScaleThreads = 512, kScaleAhead = 8;

template <int CAP>
__global__ void __launch_bounds__(kScaleThreads)
    adamw_scale_kernel(const __grid_constant__ Table<CAP> t, const float2* __restrict__ part,
                       float clip_frac, float* __restrict__ scales) {
    const int k = blockIdx.x, end = t.first[k + 1];
    TwoSum w, x;
    for (int c = t.first[k] + threadIdx.x; c < end; c += kScaleThreads * kScaleAhead) {
        float2 p[kScaleAhead];
#pragma unroll
        for (int i = 0; i < kScaleAhead; ++i)
            p[i] = c + i * kScaleThreads < end ? part[c + i * kScaleThreads] : make_float2(0.f, 0.f);
        int wide = 0;  // (one branch for all of them)
#pragma unroll
        for (int i = 0; i < kScaleAhead; ++i) wide |= __float_as_int(p[i].x) | __float_as_int(p[i].y);
        if (wide >= 0) {
#pragma unroll
            for (int i = 0; i < kScaleAhead; ++i) {
                w.add(p[i].x);
                x.add(p[i].y);
            }
        } else {
            for (int i = 0; i < kScaleAhead; ++i) {
                w.add_word(p[i].x);
                x.add_word(p[i].y);
            }
        }
    }
    double ww = w.value(), xx = x.value();
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
        ww += __shfl_xor_sync(0xffffffffu, ww, o);
        xx += __shfl_xor_sync(0xffffffffu, xx, o);
    }
    __shared__ double sh[2][kScaleThreads / 32];
    if ((threadIdx.x & 31) == 0) {
        sh[0][threadIdx.x / 32] = ww;
        sh[1][threadIdx.x / 32] = xx;
    }
    __syncthreads();
    if (threadIdx.x != 0) return;
    ww = xx = 0.0;
    for (int q = 0; q < kScaleThreads / 32; ++q) {
        ww += sh[0][q];
        xx += sh[1][q];
    }
    const double lim = static_cast<double>(clip_frac) * sqrt(ww);
    scales[k] = static_cast<float>(sqrt(xx) > lim ? lim / sqrt(xx) : 1.0);
}

// out[i] = the value of an 8-bit moment (exact in bf16: 4 significant bits times a power of two).
// Bound: HBM.
constexpr int kValueQuads = 4, kValueWarp = 128 * kValueQuads, kValueChunk = kThreads / 32 * kValueWarp;

template <bool kSigned, typename Out>
__global__ void __launch_bounds__(kThreads)
    state_values_kernel(const uint8_t* __restrict__ codes, const float* __restrict__ scales,
                        long long n, Out* __restrict__ out) {
    const long long i0 = blockIdx.x * static_cast<long long>(kValueChunk) + threadIdx.x / 32 * kValueWarp;
    if (i0 >= n) return;
    const long long i1 = i0 + 4 * (threadIdx.x & 31);
    const bool full = i0 + kValueWarp <= n;
    uint32_t c[kValueQuads];
    float scale[kValueQuads / 2];
#pragma unroll
    for (int q = 0; q < kValueQuads; ++q)
        c[q] = full ? load_codes<true>(codes, i1 + 128 * q, n) : load_codes<false>(codes, i1 + 128 * q, n);
#pragma unroll
    for (int b = 0; b < kValueQuads / 2; ++b)
        scale[b] = i0 + kAdamBlock * b < n ? scales[i0 / kAdamBlock + b] : 0.f;
#pragma unroll
    for (int q = 0; q < kValueQuads; ++q) {
        float x[4];
        from_codes<kSigned>(c[q], scale[q / 2], x);
        if (full)
            store4<true>(out, i1 + 128 * q, n, x);
        else
            store4<false>(out, i1 + 128 * q, n, x);
    }
}

template <bool kState8>
long long chunks_of(long long n) {
    return (n + Share<kState8>::kChunk - 1) / Share<kState8>::kChunk;
}

// Tensors ids[0, count) of the call, all with the same kind of state.
template <int CAP, bool kState8>
cudaError_t run_adamw(const int* ids, int count, const AdamTensor* ts, const AdamRates& op,
                      uint32_t key, float2* part, float* scales, cudaStream_t st) {
    Table<CAP> t = {};
    long long total = 0;
    for (int k = 0; k < count; ++k) {
        const AdamTensor& a = ts[ids[k]];
        t.g[k] = a.G;
        t.w[k] = a.W;
        t.wo[k] = a.W_out;
        t.m[k] = a.m;
        t.v[k] = a.v;
        t.ms[k] = a.m_scale;
        t.vs[k] = a.v_scale;
        t.n[k] = a.n;
        t.first[k] = static_cast<int>(total);
        t.key[k] = mix(key + static_cast<uint32_t>(ids[k]));
        t.wd[k] = a.weight_decay;
        t.flags[k] = static_cast<uint8_t>((a.g_bf16 ? kG16 : 0) | (a.out_bf16 ? kOut16 : 0));
        total += chunks_of<kState8>(a.n);
        if (total > 0x7fffffff) return cudaErrorInvalidValue;
    }
    t.count = count;
    t.first[count] = static_cast<int>(total);
    if (total == 0) return cudaSuccess;
    const unsigned grid = static_cast<unsigned>(total);
    float2* const no_part = nullptr;
    const float* const no_scales = nullptr;
    if (op.clip == 0)
        return launch_plain(adamw_kernel<CAP, kStep, kState8>, grid, kThreads, st, t, op, no_part, no_scales);
    constexpr Pass kFirst = kState8 ? kNorms : kMoments, kLast = kState8 ? kStep : kApply;
    cudaError_t e = op.clip == 1
        ? launch_plain(adamw_kernel<CAP, kFirst, kState8>, grid, kThreads, st, t, op, part, no_scales)
        : launch_plain(adamw_kernel<CAP, kNorms, kState8>, grid, kThreads, st, t, op, part, no_scales);
    if (e != cudaSuccess) return e;
    e = launch_plain(adamw_scale_kernel<CAP>, static_cast<unsigned>(count), kScaleThreads, st, t, part,
                     op.clip_frac, scales);
    if (e != cudaSuccess) return e;
    return op.clip == 1
        ? launch_plain(adamw_kernel<CAP, kLast, kState8>, grid, kThreads, st, t, op, no_part, scales)
        : launch_plain(adamw_kernel<CAP, kStep, kState8>, grid, kThreads, st, t, op, no_part, scales);
}

// Tensors of one launch: the table of a few is a tenth of the parameters of many.
constexpr int kFew = 12, kMany = 128;

template <bool kState8>
cudaError_t run_kind(int n_tensors, const AdamTensor* ts, const AdamRates& op, uint32_t key, float* ws,
                     cudaStream_t st) {
    float2* part = reinterpret_cast<float2*>(ws ? ws + kMany : nullptr);
    int ids[kMany], count = 0;
    for (int k = 0; k <= n_tensors; ++k) {
        if (k < n_tensors && ts[k].state8 == kState8 && ts[k].n > 0) ids[count++] = k;
        if (count < kMany && (k < n_tensors || count == 0)) continue;
        const cudaError_t e =
            count <= kFew ? run_adamw<kFew, kState8>(ids, count, ts, op, key, part, ws, st)
                          : run_adamw<kMany, kState8>(ids, count, ts, op, key, part, ws, st);
        if (e != cudaSuccess) return e;
        count = 0;
    }
    return cudaSuccess;
}

}  // namespace

size_t adamw_workspace_floats(int n_tensors, const int64_t* n) {
    // the scales of a launch's tensors, then its chunks' sums (at most those of all tensors)
    long long all = 0;
    for (int k = 0; k < n_tensors; ++k) all += chunks_of<true>(n[k]);  // (the smaller chunks)
    return static_cast<size_t>(kMany + 2 * all);
}

cudaError_t launch_adamw(int n_tensors, const AdamTensor* ts, const AdamRates& op, uint64_t seed,
                         int64_t step, float* ws, cudaStream_t st) {
    uint32_t key = mix(static_cast<uint32_t>(seed) + kPhi);
    key = mix(key ^ static_cast<uint32_t>(seed >> 32));
    key = mix(key ^ static_cast<uint32_t>(step));
    const cudaError_t e = run_kind<false>(n_tensors, ts, op, key, ws, st);
    return e != cudaSuccess ? e : run_kind<true>(n_tensors, ts, op, key, ws, st);
}

cudaError_t launch_state_values(bool is_signed, long long n, const void* codes, const float* scales,
                                int out_dtype, void* out, cudaStream_t st) {
    const long long blocks = (n + kValueChunk - 1) / kValueChunk;
    if (blocks > 0x7fffffff) return cudaErrorInvalidValue;
    const unsigned grid = static_cast<unsigned>(blocks);
    const uint8_t* c = static_cast<const uint8_t*>(codes);
    auto run = [&](auto kern, auto* to) { return launch_plain(kern, grid, kThreads, st, c, scales, n, to); };
    if (out_dtype == 1) {
        __nv_bfloat16* const to = static_cast<__nv_bfloat16*>(out);
        return is_signed ? run(state_values_kernel<true, __nv_bfloat16>, to)
                         : run(state_values_kernel<false, __nv_bfloat16>, to);
    }
    float* const to = static_cast<float*>(out);
    return is_signed ? run(state_values_kernel<true, float>, to) : run(state_values_kernel<false, float>, to);
}

}  // namespace fpo
