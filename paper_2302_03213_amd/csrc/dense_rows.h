// Products of the dense layers that are too small for tiles of laid-out operands: dense_rows.hip.
#pragma once
#include "dense_epilogue.h"

namespace lutnn {

// Up to this many rows go through the kernel for single tokens.
constexpr int kFewRows = 4;

// Y = act(X W + b) + R for N <= kFewRows rows.
hipError_t launch_few_rows(int dtype, const void* X, int64_t N, int64_t ldx, const void* W, int64_t ldw, int D, int M,
                           const Epilogue& e, hipStream_t s);

// C[i][j] = sum_k A(i, k) B(k, j) of fp32 operands as they are, the value at outer index o and k being p[o * outer + k * inner];
// one of the two steps is 1.
struct PlainOperand {
    const float* p;
    int64_t outer, inner;
};
hipError_t launch_plain_f32(const PlainOperand& A, const PlainOperand& B, int64_t I, int J, int64_t K, const Epilogue& e, hipStream_t s);

// us, as measured
float plain_f32_us(int64_t I, int J, int64_t K);

}  // namespace lutnn
