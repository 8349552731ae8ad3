// Linear layers that are not looked up: Y = act(X W + b) + R, and the gradients of X, W and b.
//
//   Z = X W + b,  Y = act(Z) + R;      dZ = dL/dY act'(Z),  dX = dZ W^T,  dW = X^T dZ,  db = sum over rows of dZ
#include "activation.h"
#include "lutnn_kernels.h"
#include "matrix_types.h"

namespace lutnn {
namespace {

constexpr int kTile = 64, kDepth = 16;

struct Epilogue {
    const float* bias;
    int activation;
    const void* R;
    void* Y;
    void* Z;
    int64_t ldr, ldy, ldz;
};

// C[i][j] = sum_k A[i * ai + k * ak] * B[k * bk + j * bj]
template <class T>
__global__ __launch_bounds__(256) void product_kernel(const T* __restrict__ A, int64_t ai, int64_t ak, const T* __restrict__ B,
                                                      int64_t bk, int64_t bj, int64_t I, int J, int64_t K, int j_tiles,
                                                      Epilogue e) {
    __shared__ float a[kDepth][kTile + 4], b[kDepth][kTile + 4];
    const int64_t i0 = (int64_t)(blockIdx.x / j_tiles) * kTile;
    const int j0 = (int)(blockIdx.x % j_tiles) * kTile;
    const int ti = threadIdx.x / 16 * 4, tj = threadIdx.x % 16 * 4;
    float sum[4][4] = {};
    for (int64_t k0 = 0; k0 < K; k0 += kDepth) {
        for (int v = threadIdx.x; v < kTile * kDepth; v += 256) {
            const int ia = ak == 1 ? v / kDepth : v % kTile, ka = ak == 1 ? v % kDepth : v / kTile;
            a[ka][ia] = i0 + ia < I && k0 + ka < K ? (float)A[(i0 + ia) * ai + (k0 + ka) * ak] : 0.f;
            const int jb = bk == 1 ? v / kDepth : v % kTile, kb = bk == 1 ? v % kDepth : v / kTile;
            b[kb][jb] = j0 + jb < J && k0 + kb < K ? (float)B[(k0 + kb) * bk + (j0 + jb) * bj] : 0.f;
        }
        __syncthreads();
#pragma unroll
        for (int k = 0; k < kDepth; ++k)
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j) sum[i][j] = __fmaf_rn(a[k][ti + i], b[k][tj + j], sum[i][j]);
        __syncthreads();
    }
    for (int i = 0; i < 4; ++i)
        for (int j = 0; j < 4; ++j) {
            const int64_t n = i0 + ti + i;
            const int m = j0 + tj + j;
            if (n >= I || m >= J) continue;
            const float z = sum[i][j] + (e.bias ? e.bias[m] : 0.f);
            if (e.Z) static_cast<T*>(e.Z)[n * e.ldz + m] = (T)z;
            const float r = e.R ? (float)static_cast<const T*>(e.R)[n * e.ldr + m] : 0.f;
            static_cast<T*>(e.Y)[n * e.ldy + m] = (T)(activate(z, e.activation) + r);
        }
}

template <class T>
hipError_t product(const T* A, int64_t ai, int64_t ak, const T* B, int64_t bk, int64_t bj, int64_t I, int J, int64_t K,
                   const Epilogue& e, hipStream_t s) {
    const int64_t j_tiles = (J + kTile - 1) / kTile, blocks = j_tiles * ((I + kTile - 1) / kTile);
    if (blocks > 0x7fffffffLL) return hipErrorInvalidValue;
    hipLaunchKernelGGL(product_kernel<T>, dim3((unsigned)blocks), dim3(256), 0, s, A, ai, ak, B, bk, bj, I, J, K, (int)j_tiles, e);
    return hipGetLastError();
}

// dZ = G act'(Z)
template <class T>
__global__ __launch_bounds__(256) void slope_kernel(const T* __restrict__ G, int64_t ldg, const T* __restrict__ Z, int64_t ldz,
                                                    int64_t N, int M, int activation, T* __restrict__ dZ) {
    for (int64_t v = blockIdx.x * 256LL + threadIdx.x; v < N * M; v += gridDim.x * 256LL) {
        const int64_t n = v / M;
        const int m = (int)(v - n * M);
        dZ[v] = (T)((float)G[n * ldg + m] * slope((float)Z[n * ldz + m], activation));
    }
}

// grid: columns / 32
template <class T>
__global__ __launch_bounds__(256) void bias_sums_kernel(const T* __restrict__ G, int64_t ldg, const T* __restrict__ Z, int64_t ldz,
                                                        int64_t N, int M, int activation, float* __restrict__ db) {
    __shared__ double part[8][32];
    const int i = threadIdx.x & 31, group = threadIdx.x >> 5, m = blockIdx.x * 32 + i;
    double sum = 0;
    if (m < M)
        for (int64_t n = group; n < N; n += 8)
            sum += (float)G[n * ldg + m] * (activation ? slope((float)Z[n * ldz + m], activation) : 1.f);
    part[group][i] = sum;
    __syncthreads();
    if (group != 0 || m >= M) return;
    for (int k = 1; k < 8; ++k) sum += part[k][i];
    db[m] = (float)sum;
}

}  // namespace

size_t dense_linear_workspace(const DenseCall&) { return 0; }

hipError_t launch_dense_linear(const DenseCall& c, const float* bias, int activation, const void* R, int64_t ldr, void* Y,
                               int64_t ldy, void* Z, int64_t ldz, void*, hipStream_t s) {
    return with_type(c.dtype, [&](auto t) {
        using T = decltype(t);
        return product(static_cast<const T*>(c.X), c.ldx, 1, static_cast<const T*>(c.W), c.ldw, 1, c.N, c.M, c.D,
                       Epilogue{bias, activation, R, Y, Z, ldr, ldy, ldz}, s);
    });
}

size_t dense_linear_gradient_workspace(const DenseCall& c, const void*, int64_t, const void*, int64_t, int activation, bool, bool, bool) {
    return activation ? (size_t)c.N * c.M * (c.dtype ? 2 : 4) : 0;
}

hipError_t launch_dense_linear_gradient(const DenseCall& c, const void* G, int64_t ldg, const void* Z, int64_t ldz, int activation,
                                        void* dX, int64_t lddx, void* dW, int64_t lddw, float* db, void* workspace,
                                        hipStream_t s) {
    return with_type(c.dtype, [&](auto t) {
        using T = decltype(t);
        const T *g = static_cast<const T*>(G), *z = static_cast<const T*>(Z);
        if (db)
            hipLaunchKernelGGL(bias_sums_kernel<T>, dim3((c.M + 31) / 32), dim3(256), 0, s, g, ldg, z, ldz, c.N, c.M, activation, db);
        if (activation && (dX || dW) && c.N > 0) {
            T* const dz = static_cast<T*>(workspace);
            hipLaunchKernelGGL(slope_kernel<T>, dim3(2048), dim3(256), 0, s, g, ldg, z, ldz, c.N, c.M, activation, dz);
            g = dz;
            ldg = c.M;
        }
        if (hipError_t e = hipGetLastError()) return e;
        const Epilogue to_x{nullptr, 0, nullptr, dX, nullptr, 0, lddx, 0}, to_w{nullptr, 0, nullptr, dW, nullptr, 0, lddw, 0};
        if (dX && c.N > 0)
            if (hipError_t e = product(g, ldg, 1, static_cast<const T*>(c.W), 1, c.ldw, c.N, c.D, c.M, to_x, s)) return e;
        if (!dW) return hipSuccess;
        return product(static_cast<const T*>(c.X), 1, c.ldx, g, ldg, 1, c.D, c.M, c.N, to_w, s);
    });
}

}  // namespace lutnn
