// act_math.cuh -- the activations of a linear layer and their derivatives.
//
//   relu       max(z, 0)                     slope 1 for z > 0, else 0
//   gelu       z Phi(z)                      Phi + z phi, Phi(z) = erfc(-z / sqrt 2) / 2
//   gelu tanh  z s(2 u)                      s + z s (1 - s) 2 u',  u = sqrt(2 / pi) (z + 0.044715 z^3)
//   silu       z s(z)                        s (1 + z (1 - s)),     s the logistic function
// (0.5 (1 + tanh u) is s(2 u), which keeps its digits where 1 + tanh u cancels.)
//
// For gelu both forms take
//   erfc(x) = exp(-x^2) t Q(t),  t = 1 / (1 + 0.38 x),  x >= 0,
// Q the polynomial that fits exp(x^2) erfc(x) / t best relative to it (over [0, 14], in fp32 [0, 10]) by iterated
// reweighted least squares; Phi(z) = erfc(|z| / sqrt 2) / 2 or 1 minus it keeps its digits in the tail.
//
// act_value and act_slope are the fp32 forms: Q of degree 8 (2e-8 off), what z^2 rounds off put back into
// the exponential, the MUFU reciprocal: z Phi within 4.8e-7 of its value over 440,000 z, 4e-8 on
// average; gelu's slope within 2.2e-7, silu's within 1e-6, gelu tanh's within 2e-6.  With erfcf, expf and a
// division the slope pass over 8192 x 1024 with gelu took 35 us instead of 27, dX of 3906 x 118 x 2602
// 121 instead of 86.
// act_value2 and act_slope2 take two values at a time where the result is rounded to bf16: packed
// f32x2 arithmetic, the MUFU exponential and reciprocal (some units of 2^-22), Q of degree 6 (1.1e-6
// off).  With erfcf the up-projection of 16384 tokens took 1135 us instead of 906 with gelu tanh: the
// epilogue's instructions cost power and issue slots beside the MMAs.
#pragma once

#include <math.h>

#include <type_traits>

namespace fpo {

enum : int { kActNone = 0, kActRelu = 1, kActGelu = 2, kActGeluTanh = 3, kActSilu = 4 };

__device__ __forceinline__ float rcp_approx(float x) {
    float y;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ float logistic(float x) {
    return rcp_approx(1.f + expf(-x));  // x < -88: exp is infinite and its reciprocal 0
}

constexpr float kGeluU = 0.7978845608028654f;   // sqrt(2 / pi)
constexpr float kGeluC = 0.044715f;
constexpr float kSqrtHalf = 0.7071067811865476f;
constexpr float kInvSqrt2Pi = 0.3989422804014327f;

// exp(-z^2 / 2) and Phi(z); beyond 16 the one is 0 and the other 0 or 1 (0 for a NaN).
__device__ __forceinline__ void normal(float z, float& e, float& cdf) {
    const float a = fminf(fabsf(z), 16.f), t = rcp_approx(fmaf(a, 0.38f * kSqrtHalf, 1.f));
    const float h = a * a, rest = fmaf(a, a, -h);
    e = expf(-0.5f * h);
    e = fmaf(e, -0.5f * rest, e);
    float q = fmaf(t, 0.0589897118f, -0.26239594f);
    q = fmaf(t, q, 0.364107609f);
    q = fmaf(t, q, -0.161752464f);
    q = fmaf(t, q, 0.230237057f);
    q = fmaf(t, q, 0.138554962f);
    q = fmaf(t, q, 0.203932415f);
    q = fmaf(t, q, 0.213915459f);
    q = fmaf(t, q, 0.21441121f);
    const float tail = 0.5f * t * (q * e);  // Phi(-|z|)
    cdf = z > 0.f ? 1.f - tail : tail;
}

template <int kAct>
__device__ __forceinline__ float act_value(float z) {
    if constexpr (kAct == kActRelu) return z < 0.f ? 0.f : z;  // (NaN stays)
    if constexpr (kAct == kActGelu) {
        float e, cdf;
        normal(z, e, cdf);
        return z * cdf;
    }
    if constexpr (kAct == kActGeluTanh)
        return z * logistic(2.f * kGeluU * z * fmaf(kGeluC * z, z, 1.f));
    if constexpr (kAct == kActSilu) return z * logistic(z);
    return z;
}

template <int kAct>
__device__ __forceinline__ float act_slope(float z) {
    if constexpr (kAct == kActRelu) return z > 0.f ? 1.f : 0.f;
    if constexpr (kAct == kActGelu) {
        float e, cdf;
        normal(z, e, cdf);
        return fmaf(z, kInvSqrt2Pi * e, cdf);
    }
    if constexpr (kAct == kActGeluTanh) {
        // beyond 12 the slope is 0 or 1 to fp32, and z^2 could overflow against s (1 - s) = 0
        if (fabsf(z) > 12.f) return z > 0.f ? 1.f : 0.f;
        const float q = kGeluC * z * z;
        const float s = logistic(2.f * kGeluU * fmaf(z, q, z));
        return fmaf(z * s * (1.f - s), 2.f * kGeluU * fmaf(3.f, q, 1.f), s);
    }
    if constexpr (kAct == kActSilu) {
        const float s = logistic(z);
        return s * fmaf(z, 1.f - s, 1.f);
    }
    return 1.f;
}

// ------------------------------------------------------------------ two values, for bf16 results
__device__ __forceinline__ float2 both(float x) { return make_float2(x, x); }
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c) { return __ffma2_rn(a, b, c); }
__device__ __forceinline__ float2 mul2(float2 a, float2 b) { return __fmul2_rn(a, b); }
__device__ __forceinline__ float2 add2(float2 a, float2 b) { return __fadd2_rn(a, b); }
__device__ __forceinline__ float exp2_approx(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

constexpr float kLog2E = 1.4426950408889634f;

// 1 / (1 + 2^x): the logistic function of -x log 2.
__device__ __forceinline__ float2 logistic_exp2(float2 x) {
    const float2 d = add2(make_float2(exp2_approx(x.x), exp2_approx(x.y)), both(1.f));
    return make_float2(rcp_approx(d.x), rcp_approx(d.y));
}
// exp(-z^2 / 2) and Phi(z).
__device__ __forceinline__ void normal2(float2 z, float2& e, float2& cdf) {
    const float2 a = make_float2(fabsf(z.x), fabsf(z.y));
    const float2 d = fma2(a, both(0.38f * kSqrtHalf), both(1.f));
    const float2 t = make_float2(rcp_approx(d.x), rcp_approx(d.y));
    const float2 x = mul2(mul2(z, both(-0.5f * kLog2E)), z);
    e = make_float2(exp2_approx(x.x), exp2_approx(x.y));
    float2 q = fma2(t, both(-0.12542358f), both(0.33605671f));
    q = fma2(t, q, both(-0.06994075f));
    q = fma2(t, q, both(0.24785321f));
    q = fma2(t, q, both(0.18058746f));
    q = fma2(t, q, both(0.21657866f));
    q = fma2(t, q, both(0.21428722f));
    const float2 tail = mul2(mul2(t, both(0.5f)), mul2(q, e));  // Phi(-|z|)
    cdf = make_float2(z.x > 0.f ? 1.f - tail.x : tail.x, z.y > 0.f ? 1.f - tail.y : tail.y);
}

template <int kAct>
__device__ __forceinline__ float2 act_value2(float2 z) {
    if constexpr (kAct == kActRelu) return make_float2(z.x < 0.f ? 0.f : z.x, z.y < 0.f ? 0.f : z.y);
    if constexpr (kAct == kActGelu) {
        float2 e, cdf;
        normal2(z, e, cdf);
        return mul2(z, cdf);
    }
    if constexpr (kAct == kActGeluTanh) {
        constexpr float k = -2.f * kGeluU * kLog2E;
        return mul2(z, logistic_exp2(mul2(z, fma2(mul2(z, both(k * kGeluC)), z, both(k)))));
    }
    if constexpr (kAct == kActSilu) return mul2(z, logistic_exp2(mul2(z, both(-kLog2E))));
    return z;
}

template <int kAct>
__device__ __forceinline__ float2 act_slope2(float2 z) {
    if constexpr (kAct == kActRelu) return make_float2(z.x > 0.f ? 1.f : 0.f, z.y > 0.f ? 1.f : 0.f);
    if constexpr (kAct == kActGelu) {
        float2 e, cdf;
        normal2(z, e, cdf);
        return fma2(mul2(z, both(kInvSqrt2Pi)), e, cdf);
    }
    if constexpr (kAct == kActGeluTanh) {
        constexpr float k = -2.f * kGeluU * kLog2E;
        const float2 q = mul2(mul2(z, both(kGeluC)), z);
        const float2 s = logistic_exp2(mul2(mul2(z, both(k)), add2(q, both(1.f))));
        const float2 u = mul2(z, fma2(q, both(6.f * kGeluU), both(2.f * kGeluU)));
        const float2 r = fma2(mul2(s, add2(both(1.f), make_float2(-s.x, -s.y))), u, s);
        // beyond 12 it is 0 or 1, and z^2 could overflow against s (1 - s) = 0
        return make_float2(fabsf(z.x) > 12.f ? (z.x > 0.f ? 1.f : 0.f) : r.x,
                           fabsf(z.y) > 12.f ? (z.y > 0.f ? 1.f : 0.f) : r.y);
    }
    if constexpr (kAct == kActSilu) {
        const float2 s = logistic_exp2(mul2(z, both(-kLog2E)));
        return mul2(s, fma2(z, add2(both(1.f), make_float2(-s.x, -s.y)), both(1.f)));
    }
    return both(1.f);
}

// f(std::integral_constant<int, act>): one branch around a loop over elements.
template <class F>
__device__ __forceinline__ void with_act(int act, F&& f) {
    switch (act) {
        case kActRelu: f(std::integral_constant<int, kActRelu>{}); break;
        case kActGelu: f(std::integral_constant<int, kActGelu>{}); break;
        case kActGeluTanh: f(std::integral_constant<int, kActGeluTanh>{}); break;
        case kActSilu: f(std::integral_constant<int, kActSilu>{}); break;
        default: f(std::integral_constant<int, kActNone>{}); break;
    }
}

}  // namespace fpo
