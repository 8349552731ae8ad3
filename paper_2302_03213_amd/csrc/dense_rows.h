// Products of the dense layers that are too small for tiles of laid-out operands: dense_rows.hip.
#pragma once
#include "dense_epilogue.h"

namespace lutnn {

// Tiles of a product: a launch has 2^32 threads at most.
constexpr int64_t kMostTiles = 1 << 21;

// Whether N rows go through the kernel for single tokens.  fp32: four rows of 4096 x 4096 14 us, eight 17, five to sixteen by tiles
// 23; eight of 1024 x 4096 8.0 and 7.7, of 4096 x 512 11 and 17, of 8192 x 1024 18.8 and 17.9.  16 bits: one row of 1024 x 4096 5.4,
// two 6.3, four 8.4, two to sixteen by tiles 6.8; of 4096 x 4096 12.0, 13.5, 16.2 and 11.7.
constexpr int most_few_rows(int dtype) { return dtype == 0 ? 8 : 2; }
inline bool few_rows(int dtype, int64_t N, int D, int M) {
    const bool large = (int64_t)D * M >= 1 << 23;
    return N <= (dtype == 0 ? (large || D >= 2048 ? 8 : 4) : (large ? 1 : 2));
}

// Y = act(X W + b) + R for so many.
hipError_t launch_few_rows(int dtype, const void* X, int64_t N, int64_t ldx, const void* W, int64_t ldw, int D, int M,
                           const Epilogue& e, hipStream_t s);

// Rows to be added up by workgroups of a launch beside other work: fp32 sums that an earlier kernel's workgroups left,
// [count][width], or a matrix of the launch's type itself, row stride ld; no `out`: none.
struct PartialSums {
    const float* partial;
    int count, width;
    float* out;
    const void* matrix;
    int64_t ld;
};

// 32 columns of them by workgroup `block` of THREADS, 64-bit sums in a fixed order.  lds: THREADS / 32 * 33 doubles.
template <class T, int THREADS>
__device__ __forceinline__ void add_partial_sums(const PartialSums& p, int block, void* lds) {
    constexpr int GROUPS = THREADS / 32;
    double(*const part)[33] = static_cast<double(*)[33]>(lds);
    const int i = threadIdx.x & 31, group = threadIdx.x >> 5, m = block * 32 + i;
    double sum = 0;
    const auto add = [&](const auto* from, int64_t ld) {
#pragma unroll 8
        for (int k = group; k < p.count; k += GROUPS) sum += (float)from[k * ld + m];
    };
    if (m < p.width) {
        if (p.matrix)
            add(static_cast<const T*>(p.matrix), p.ld);
        else
            add(p.partial, p.width);
    }
    part[group][i] = sum;
    __syncthreads();
    if (group != 0 || m >= p.width) return;
#pragma unroll
    for (int k = 1; k < GROUPS; ++k) sum += part[k][i];
    p.out[m] = (float)sum;
}

// C[i][j] = sum_k A(i, k) B(k, j) of fp32 operands as they are, the value at outer index o and k being p[o * outer + k * inner];
// one of the two steps is 1.
struct PlainOperand {
    const float* p;
    int64_t outer, inner;
};
hipError_t launch_plain_f32(const PlainOperand& A, const PlainOperand& B, int64_t I, int J, int64_t K, const Epilogue& e, hipStream_t s);

// dX [I][J] and dW [WI][WJ] in one launch, with the partial sums added up beside them: dX = dZ W^T, dW = X^T dZ.
hipError_t launch_plain_pair_f32(const float* dZ, int64_t ldg, const float* W, int64_t ldw, const float* X, int64_t ldx, int64_t N, int D,
                                 int M, const Epilogue& to_x, const Epilogue& to_w, const PartialSums& sums, hipStream_t s);
float plain_pair_us(int64_t N, int D, int M);

// us, as measured
float plain_f32_us(int64_t I, int J, int64_t K);

}  // namespace lutnn
