// The activations of a dense linear layer's epilogue and their slopes, in fp32.
#pragma once
#include <hip/hip_runtime.h>

#include <type_traits>

namespace lutnn {

enum Activation { kActNone = 0, kActRelu, kActGelu, kActGeluTanh, kActSilu };

// 1 / (1 + exp(-z)); 0 and 1 where exp leaves its range
__device__ __forceinline__ float logistic(float z) { return __builtin_amdgcn_rcpf(1.f + __expf(-z)); }

// The normal distribution's upper tail beyond |z|, and exp(-z^2 / 2) beside it: erfc(x) = t (a1 + t (a2 + ...)) exp(-x^2) with
// t = 1 / (1 + p x), x = |z| / sqrt 2, within 1.5e-7 (M. Abramowitz, I. Stegun, Handbook of Mathematical Functions, 7.1.26, after
// C. Hastings).  A third of erff's instructions, which a tile of a product has nothing to hide behind.
__device__ __forceinline__ float normal_tail(float z, float& density) {
    const float t = __builtin_amdgcn_rcpf(__fmaf_rn(0.3275911f * 0.70710678118654752f, fabsf(z), 1.f));
    density = __builtin_amdgcn_exp2f(z * z * -0.72134752044448170f);  // log2(e) / 2
    const float sum = __fmaf_rn(t, __fmaf_rn(t, __fmaf_rn(t, __fmaf_rn(t, 0.5f * 1.061405429f, 0.5f * -1.453152027f), 0.5f * 1.421413741f),
                                             0.5f * -0.284496736f), 0.5f * 0.254829592f);
    return sum * t * density;
}

// gelu's approximation by tanh is z logistic(2 u): (1 + tanh u) / 2 = logistic(2 u)
constexpr float kGeluTanhScale = 2.f * 0.7978845608028654f;  // 2 sqrt(2 / pi)
constexpr float kGeluTanhCubic = 0.044715f;

__device__ __forceinline__ float activate(float z, int activation) {
    switch (activation) {
        case kActRelu: return z < 0.f ? 0.f : z;
        case kActGelu: {
            float density;  // z Phi(z) = max(z, 0) - |z| Phi(-|z|), where the last is a zero long before |z| reaches 100
            const float tail = normal_tail(z, density);
            return __fmaf_rn(-fminf(fabsf(z), 100.f), tail, fmaxf(z, 0.f));
        }
        case kActGeluTanh: return z * logistic(kGeluTanhScale * z * (1.f + kGeluTanhCubic * z * z));
        case kActSilu: return z * logistic(z);
        default: return z;
    }
}

// Far from zero 0 or 1, also where a product below would be of an infinite z, or z * z, and a zero.
__device__ __forceinline__ float slope(float z, int activation) {
    if (fabsf(z) > (activation == kActSilu ? 90.f : 30.f)) return z > 0.f ? 1.f : 0.f;
    switch (activation) {
        case kActRelu: return z > 0.f ? 1.f : 0.f;
        case kActGelu: {
            float density;
            const float tail = normal_tail(z, density);
            return __fmaf_rn(z * 0.3989422804014327f, density, z < 0.f ? tail : 1.f - tail);
        }
        case kActGeluTanh: {
            const float zz = z * z, s = logistic(kGeluTanhScale * z * (1.f + kGeluTanhCubic * zz));
            return s + z * s * (1.f - s) * kGeluTanhScale * (1.f + 3.f * kGeluTanhCubic * zz);
        }
        case kActSilu: {
            const float s = logistic(z);
            return s * (1.f + z * (1.f - s));
        }
        default: return 1.f;
    }
}

// Calls f with the activation as a constant; not at all for none.
template <class F>
__device__ __forceinline__ void with_activation(int activation, F&& f) {
    switch (activation) {
        case kActRelu: return f(std::integral_constant<int, kActRelu>());
        case kActGelu: return f(std::integral_constant<int, kActGelu>());
        case kActGeluTanh: return f(std::integral_constant<int, kActGeluTanh>());
        case kActSilu: return f(std::integral_constant<int, kActSilu>());
    }
}

// g times the slopes at z
template <int n>
__device__ __forceinline__ void slope_all(float (&g)[n], const float (&z)[n], int activation) {
    with_activation(activation, [&](auto kind) {
#pragma unroll
        for (int r = 0; r < n; ++r) g[r] *= slope(z[r], decltype(kind)::value);
    });
}

}  // namespace lutnn
