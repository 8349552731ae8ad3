// The activations of a dense linear layer's epilogue and their slopes, in fp32.
#pragma once
#include <hip/hip_runtime.h>

#include <type_traits>

namespace lutnn {

enum Activation { kActNone = 0, kActRelu, kActGelu, kActGeluTanh, kActSilu };

// 1 / (1 + exp(-z)); 0 and 1 where exp leaves its range
__device__ __forceinline__ float logistic(float z) { return __builtin_amdgcn_rcpf(1.f + __expf(-z)); }

// gelu's approximation by tanh is z logistic(2 u): (1 + tanh u) / 2 = logistic(2 u)
constexpr float kGeluTanhScale = 2.f * 0.7978845608028654f;  // 2 sqrt(2 / pi)
constexpr float kGeluTanhCubic = 0.044715f;

__device__ __forceinline__ float activate(float z, int activation) {
    switch (activation) {
        case kActRelu: return z < 0.f ? 0.f : z;
        case kActGelu: return 0.5f * z * (1.f + erff(z * 0.70710678118654752f));
        case kActGeluTanh: return z * logistic(kGeluTanhScale * z * (1.f + kGeluTanhCubic * z * z));
        case kActSilu: return z * logistic(z);
        default: return z;
    }
}

__device__ __forceinline__ float slope(float z, int activation) {
    switch (activation) {
        case kActRelu: return z > 0.f ? 1.f : 0.f;
        case kActGelu: return 0.5f * (1.f + erff(z * 0.70710678118654752f)) + z * 0.3989422804014327f * __expf(-0.5f * z * z);
        case kActGeluTanh: {
            if (fabsf(z) > 30.f) return z > 0.f ? 1.f : 0.f;  // where z * z may overflow against a zero
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

template <int n>
__device__ __forceinline__ void activate_all(float (&z)[n], int activation) {
    with_activation(activation, [&](auto kind) {
#pragma unroll
        for (int r = 0; r < n; ++r) z[r] = activate(z[r], decltype(kind)::value);
    });
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
