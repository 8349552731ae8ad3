// Dense layers of few rows: what bounds them is reading W once and the launch itself, so each is one launch that reads its operands
// as they are.
#include <algorithm>
#include <type_traits>

#include "dense_rows.h"
#include "lutnn_kernels.h"

namespace lutnn {
namespace {

constexpr int kThreads = 512, kWaves = kThreads / 64;
constexpr int kCols = 16;  // of a workgroup

// Workgroup b's strip of columns: contiguous ranges on each XCD, as the strips of one 128-byte line of W share its L2.
__device__ __forceinline__ int strip_of(int b, int strips) {
    const int t = (b & 7) * ((strips + 7) / 8) + (b >> 3);
    return t < strips ? t : -1;
}

// A strip of 16 columns per workgroup.  A lane reads 16 bytes of a row of W, 2 (fp32: 4) lanes a row, and a workgroup 256 (128) rows
// at a time, AHEAD times that in flight; the sums over k stay in the lane to the end, and go through the wavefront and LDS then.
// grid: strips.
template <class T, int ROWS>
__global__ __launch_bounds__(kThreads) void few_rows_kernel(const T* __restrict__ X, int N, int64_t ldx, const T* __restrict__ W,
                                                            int64_t ldw, int D, int M, int strips, Epilogue e) {
    constexpr int V = 16 / sizeof(T), LANES = kCols / V, STEP = kThreads / LANES, AHEAD = 4;
    __shared__ float part[kWaves][ROWS][kCols];
    const int strip = strip_of(blockIdx.x, strips);
    if (strip < 0) return;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int j = strip * kCols + lane % LANES * V;
    const bool whole = j + V <= M;
    float sum[ROWS][V] = {};
    const auto add = [&](auto count, int k0) {
        constexpr int n = decltype(count)::value;
        float w[n][V], x[n][ROWS];
#pragma unroll
        for (int a = 0; a < n; ++a) {
            const int64_t k = min(k0 + a * STEP, D - 1);  // past the last row: that one, times zero
            const T* const from = W + k * ldw + j;
            if (whole)
                load_values(from, w[a]);
            else
#pragma unroll
                for (int c = 0; c < V; ++c) w[a][c] = j + c < M ? (float)from[c] : 0.f;
#pragma unroll
            for (int r = 0; r < ROWS; ++r) x[a][r] = (float)X[min(r, N - 1) * ldx + k];
        }
#pragma unroll
        for (int a = 0; a < n; ++a)
            if (k0 + a * STEP < D)
#pragma unroll
                for (int r = 0; r < ROWS; ++r)
#pragma unroll
                    for (int c = 0; c < V; ++c) sum[r][c] = __fmaf_rn(x[a][r], w[a][c], sum[r][c]);
    };
    int k = threadIdx.x / LANES;
    for (; k + (AHEAD - 1) * STEP < D; k += AHEAD * STEP) add(std::integral_constant<int, AHEAD>(), k);
    if (k < D) add(std::integral_constant<int, AHEAD - 1>(), k);
#pragma unroll
    for (int d = LANES; d < 64; d *= 2)
#pragma unroll
        for (int r = 0; r < ROWS; ++r)
#pragma unroll
            for (int c = 0; c < V; ++c) sum[r][c] += __shfl_xor(sum[r][c], d, 64);
    if (lane < LANES)
#pragma unroll
        for (int r = 0; r < ROWS; ++r)
#pragma unroll
            for (int c = 0; c < V; ++c) part[wave][r][lane * V + c] = sum[r][c];
    __syncthreads();
    const int r = threadIdx.x / kCols, c = threadIdx.x % kCols, col = strip * kCols + c;
    if (r >= N || r >= ROWS || col >= M) return;
    float z[1][1] = {{0.f}}, bias[1];
#pragma unroll
    for (int w = 0; w < kWaves; ++w) z[0][0] += part[w][r][c];
    load_bias(e, col, M, bias);
    const int64_t row[1] = {r};
    finish<T>(e, row, col, N, M, bias, z);
}

typedef float f32x4 __attribute__((ext_vector_type(4)));

// Four consecutive k of one outer index, zeros from k_left on.
template <bool K_INNER>
__device__ __forceinline__ f32x4 four(const PlainOperand& o, int64_t outer, int64_t k, int k_left) {
    const float* const at = o.p + outer * o.outer + k * o.inner;
    f32x4 v;
    if (K_INNER && k_left >= 4) {
        float x[4];
        load_values(at, x);
        return f32x4{x[0], x[1], x[2], x[3]};
    }
#pragma unroll
    for (int r = 0; r < 4; ++r) v[r] = r < k_left ? at[r * o.inner] : 0.f;
    return v;
}

// 16 FI rows by 16 columns per workgroup on the fp32 matrix instructions; the wavefronts take every eighth 16 k, and add up in LDS.
// An instruction sums four k, one per 16 lanes: lane group q holds k = 4 q .. 4 q + 3 of both operands, and instruction r takes the
// r-th of each.  grid: row blocks * strips, row block fastest.
template <int FI, bool A_K, bool B_K>
__global__ __launch_bounds__(kThreads) void plain_f32_kernel(PlainOperand A, PlainOperand B, int64_t I, int J, int64_t K, int row_blocks,
                                                             int strips, Epilogue e) {
    constexpr int AHEAD = FI == 1 ? 4 : 2;
    __shared__ float part[kWaves][FI * 16][kCols + 1];
    const int block = strip_of(blockIdx.x, row_blocks * strips);
    if (block < 0) return;
    const int64_t i0 = (int64_t)(block % row_blocks) * FI * 16;
    const int j0 = block / row_blocks * kCols;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, i16 = lane & 15, q = lane >> 4;
    f32x4 sum[FI] = {};
    const auto add = [&](auto count, int64_t k0) {
        constexpr int n = decltype(count)::value;
        f32x4 a[n][FI], b[n];
#pragma unroll
        for (int u = 0; u < n; ++u) {
            const int64_t k = k0 + u * 16 * kWaves + 4 * q;
            const int left = (int)max((int64_t)0, min(K - k, (int64_t)4));
            const int64_t in = min(k, K - 1);
            b[u] = four<B_K>(B, min(j0 + i16, J - 1), in, left);
#pragma unroll
            for (int i = 0; i < FI; ++i) a[u][i] = four<A_K>(A, min(i0 + 16 * i + i16, I - 1), in, left);
        }
#pragma unroll
        for (int u = 0; u < n; ++u)
#pragma unroll
            for (int r = 0; r < 4; ++r)
#pragma unroll
                for (int i = 0; i < FI; ++i) sum[i] = __builtin_amdgcn_mfma_f32_16x16x4f32(b[u][r], a[u][i][r], sum[i], 0, 0, 0);
    };
    int64_t k = 16 * wave;
    for (; k + (AHEAD / 2) * 16 * kWaves < K; k += AHEAD * 16 * kWaves) add(std::integral_constant<int, AHEAD>(), k);
    if (k < K) add(std::integral_constant<int, AHEAD / 2>(), k);
    // the first operand's index is the instruction's row: a lane has columns 4 q .. 4 q + 3 of row i16
#pragma unroll
    for (int i = 0; i < FI; ++i)
#pragma unroll
        for (int r = 0; r < 4; ++r) part[wave][16 * i + i16][4 * q + r] = sum[i][r];
    __syncthreads();
    for (int v = threadIdx.x; v < FI * 16 * kCols; v += kThreads) {
        const int64_t row[1] = {i0 + v / kCols};
        const int col = j0 + v % kCols;
        if (row[0] >= I || col >= J) continue;
        float z[1][1] = {{0.f}}, bias[1];
#pragma unroll
        for (int w = 0; w < kWaves; ++w) z[0][0] += part[w][v / kCols][v % kCols];
        load_bias(e, col, J, bias);
        finish<float>(e, row, col, I, J, bias, z);
    }
}

// Row fragments per workgroup: up to four, which read a strip of W once for all of them, but a workgroup for every compute unit first.
int row_fragments(int64_t I, int J, int units) {
    const int64_t strips = (J + kCols - 1) / kCols, fragments = (I + 15) / 16;
    return (int)std::max<int64_t>(1, std::min<int64_t>(4, fragments * strips / units));
}

}  // namespace

hipError_t launch_few_rows(int dtype, const void* X, int64_t N, int64_t ldx, const void* W, int64_t ldw, int D, int M,
                           const Epilogue& e, hipStream_t s) {
    const int strips = (M + kCols - 1) / kCols;
    return with_type(dtype, [&](auto t) {
        using T = decltype(t);
        const auto launch = [&](auto rows) {
            hipLaunchKernelGGL((few_rows_kernel<T, decltype(rows)::value>), dim3((unsigned)(strips + 7) / 8 * 8), dim3(kThreads), 0, s,
                               static_cast<const T*>(X), (int)N, ldx, static_cast<const T*>(W), ldw, D, M, strips, e);
            return hipGetLastError();
        };
        if (N == 1) return launch(std::integral_constant<int, 1>());
        return N == 2 ? launch(std::integral_constant<int, 2>()) : launch(std::integral_constant<int, kFewRows>());
    });
}

hipError_t launch_plain_f32(const PlainOperand& A, const PlainOperand& B, int64_t I, int J, int64_t K, const Epilogue& e, hipStream_t s) {
    const int fragments = row_fragments(I, J, compute_units()), strips = (J + kCols - 1) / kCols;
    const int64_t row_blocks = (I + 16 * fragments - 1) / (16 * fragments);
    if (row_blocks * strips > (1 << 30)) return hipErrorInvalidValue;
    const auto with = [&](auto fi) {
        const auto launch = [&](auto ak, auto bk) {
            hipLaunchKernelGGL((plain_f32_kernel<decltype(fi)::value, decltype(ak)::value, decltype(bk)::value>),
                               dim3((unsigned)(row_blocks * strips + 7) / 8 * 8), dim3(kThreads), 0, s, A, B, I, J, K, (int)row_blocks,
                               strips, e);
            return hipGetLastError();
        };
        if (A.inner != 1) return launch(std::false_type(), std::false_type());
        return B.inner == 1 ? launch(std::true_type(), std::true_type()) : launch(std::true_type(), std::false_type());
    };
    switch (fragments) {
        case 1: return with(std::integral_constant<int, 1>());
        case 2: return with(std::integral_constant<int, 2>());
        case 3: return with(std::integral_constant<int, 3>());
        default: return with(std::integral_constant<int, 4>());
    }
}

// A launch, and 2.3 ns per k, fragment and round of workgroups.
float plain_f32_us(int64_t I, int J, int64_t K) {
    const int units = compute_units(), fragments = row_fragments(I, J, units);
    const int64_t blocks = ((I + 16 * fragments - 1) / (16 * fragments)) * ((J + kCols - 1) / kCols);
    return 4.f + (float)((blocks + units - 1) / units) * K * 0.0023f * (fragments + 0.25f);
}

}  // namespace lutnn
