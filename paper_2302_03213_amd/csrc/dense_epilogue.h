// What becomes of a dense layer's sums: bias, activation and residual, with the values before the activation kept on request.
#pragma once
#include "activation.h"
#include "matrix_types.h"

namespace lutnn {

struct Epilogue {
    const float* bias;
    int activation;
    const void* R;
    void* Y;
    void* Z;
    int64_t ldr, ldy, ldz;
};

// The epilogue for `rows` rows of `n` columns from j on, row r at i[r]: what is read of the residual is asked for at once.  bias:
// that of the columns, zeros without one.
template <class T, int rows, int n>
__device__ __forceinline__ void finish(const Epilogue& e, const int64_t (&i)[rows], int j, int64_t I, int J, const float (&bias)[n],
                                       float (&z)[rows][n]) {
    const bool whole = j + n <= J;
    float x[rows][n] = {};
    if (e.R) {
#pragma unroll
        for (int r = 0; r < rows; ++r) {
            const T* const from = static_cast<const T*>(e.R) + min(i[r], I - 1) * e.ldr + j;
            if (whole)
                load_values(from, x[r]);
            else
#pragma unroll
                for (int c = 0; c < n; ++c) x[r][c] = j + c < J ? (float)from[c] : 0.f;
        }
    }
    const auto store = [&](void* to, int64_t ld, const float(&v)[n], int r) {
        if (i[r] >= I) return;
        T* const at = static_cast<T*>(to) + i[r] * ld + j;
        if (whole)
            store_values(at, v);
        else
#pragma unroll
            for (int c = 0; c < n; ++c)
                if (j + c < J) at[c] = (T)v[c];
    };
#pragma unroll
    for (int r = 0; r < rows; ++r) {
#pragma unroll
        for (int c = 0; c < n; ++c) z[r][c] += bias[c];
        if (e.Z) store(e.Z, e.ldz, z[r], r);
    }
    with_activation(e.activation, [&](auto kind) {
#pragma unroll
        for (int r = 0; r < rows; ++r)
#pragma unroll
            for (int c = 0; c < n; ++c) z[r][c] = activate(z[r][c], decltype(kind)::value);
    });
#pragma unroll
    for (int r = 0; r < rows; ++r) {
#pragma unroll
        for (int c = 0; c < n; ++c) z[r][c] += x[r][c];
        store(e.Y, e.ldy, z[r], r);
    }
}

// The bias of n columns from j on, zeros past the last.
template <int n>
__device__ __forceinline__ void load_bias(const Epilogue& e, int j, int J, float (&bias)[n]) {
#pragma unroll
    for (int c = 0; c < n; ++c) bias[c] = e.bias && j + c < J ? e.bias[j + c] : 0.f;
}

}  // namespace lutnn
