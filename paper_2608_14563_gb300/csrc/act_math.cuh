// act_math.cuh -- the activations of a linear layer and their derivatives on one fp32 value.
//
//   relu       max(z, 0)                     slope 1 for z > 0, else 0
//   gelu       z Phi(z)                      Phi + z phi, Phi(z) = erfc(-z / sqrt 2) / 2
//   gelu tanh  z s(2 u)                      s + z s (1 - s) 2 u',  u = sqrt(2 / pi) (z + 0.044715 z^3)
//   silu       z s(z)                        s (1 + z (1 - s)),     s the logistic function
// (0.5 (1 + tanh u) is s(2 u), which keeps its digits where 1 + tanh u cancels).  kFast: the
// MUFU exponential and divide, a few units of 2^-23 off, where the result is rounded to bf16.
#pragma once

#include <math.h>

#include <type_traits>

namespace fpo {

enum : int { kActNone = 0, kActRelu = 1, kActGelu = 2, kActGeluTanh = 3, kActSilu = 4 };

template <bool kFast>
__device__ __forceinline__ float logistic(float x) {
    // x < -88: exp overflows to infinity and the quotient is 0
    return kFast ? __fdividef(1.f, 1.f + __expf(-x)) : 1.f / (1.f + expf(-x));
}

constexpr float kGeluU = 0.7978845608028654f;   // sqrt(2 / pi)
constexpr float kGeluC = 0.044715f;
constexpr float kSqrtHalf = 0.7071067811865476f;

template <int kAct, bool kFast>
__device__ __forceinline__ float act_value(float z) {
    if constexpr (kAct == kActRelu) return z < 0.f ? 0.f : z;  // (NaN stays)
    if constexpr (kAct == kActGelu) return 0.5f * z * erfcf(-kSqrtHalf * z);
    if constexpr (kAct == kActGeluTanh)
        return z * logistic<kFast>(2.f * kGeluU * z * fmaf(kGeluC * z, z, 1.f));
    if constexpr (kAct == kActSilu) return z * logistic<kFast>(z);
    return z;
}

template <int kAct, bool kFast>
__device__ __forceinline__ float act_slope(float z) {
    if constexpr (kAct == kActRelu) return z > 0.f ? 1.f : 0.f;
    if constexpr (kAct == kActGelu) {
        const float e = kFast ? __expf(-0.5f * z * z) : expf(-0.5f * z * z);
        return fmaf(z, 0.3989422804014327f * e, 0.5f * erfcf(-kSqrtHalf * z));
    }
    if constexpr (kAct == kActGeluTanh) {
        // beyond 12 the slope is 0 or 1 to fp32, and z^2 could overflow against s (1 - s) = 0
        if (fabsf(z) > 12.f) return z > 0.f ? 1.f : 0.f;
        const float q = kGeluC * z * z;
        const float s = logistic<kFast>(2.f * kGeluU * fmaf(z, q, z));
        return fmaf(z * s * (1.f - s), 2.f * kGeluU * fmaf(3.f, q, 1.f), s);
    }
    if constexpr (kAct == kActSilu) {
        const float s = logistic<kFast>(z);
        return s * fmaf(z, 1.f - s, 1.f);
    }
    return 1.f;
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
