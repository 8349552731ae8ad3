// The types of the dense layers' matrices (fp32, bf16, fp16) in kernels: vectors of them as they are loaded and stored, and their
// values as the fp32 that everything is computed in.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace lutnn {

typedef __bf16 bf16;
typedef _Float16 f16;

// n consecutive values, at any address that one value may have: the hardware loads and stores 16 bytes from there.
template <class T, int n>
struct Packed {
    typedef T type __attribute__((ext_vector_type(n), aligned(sizeof(T))));
};
template <class T>
struct Packed<T, 1> {
    typedef T type;
};

template <class T, int n>
__device__ __forceinline__ void load_values(const T* __restrict__ from, float (&to)[n]) {
    const typename Packed<T, n>::type v = *reinterpret_cast<const typename Packed<T, n>::type*>(from);
    if constexpr (n == 1)
        to[0] = (float)v;
    else
#pragma unroll
        for (int i = 0; i < n; ++i) to[i] = (float)v[i];
}

// Rounded to the nearest value of T, ties to even; what is beyond T becomes infinite.
template <class T, int n>
__device__ __forceinline__ void store_values(T* __restrict__ to, const float (&from)[n]) {
    typename Packed<T, n>::type v;
    if constexpr (n == 1)
        v = (T)from[0];
    else
#pragma unroll
        for (int i = 0; i < n; ++i) v[i] = (T)from[i];
    *reinterpret_cast<typename Packed<T, n>::type*>(to) = v;
}

// Calls f with a value of the type that a lutnn_dtype stands for.
template <class F>
hipError_t with_type(int dtype, F&& f) {
    if (dtype == 0) return f(float());
    return dtype == 1 ? f(bf16()) : f(f16());
}

}  // namespace lutnn
