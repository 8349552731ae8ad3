// Dense layers of few rows: what bounds them is reading W once and the launch itself, so each is one launch that reads its operands
// as they are.  1 x 1024 x 4096 in bf16 4.7 us, 8.4 MB at 1.8 TB/s; 37 x 768 x 768 in fp32 5.8.
#include <algorithm>
#include <cmath>
#include <type_traits>

#include "dense_rows.h"
#include "lutnn_kernels.h"

namespace lutnn {
namespace {

constexpr int kThreads = 512, kWaves = kThreads / 64;

// Workgroup b's strip of columns: contiguous ranges on each XCD, as the strips of one 128-byte line of W share its L2.
__device__ __forceinline__ int strip_of(int b, int strips) {
    const int t = (b & 7) * ((strips + 7) / 8) + (b >> 3);
    return t < strips ? t : -1;
}

// A strip of COLS columns per workgroup.  A lane reads 16 bytes of a row of W, 2 (fp32: 4) lanes a row of 16 columns, and a workgroup
// 256 (128) such rows at a time, AHEAD times that in flight; the sums over k stay in the lane to the end, and go through the
// wavefront and LDS then.  grid: strips.
template <class T, int ROWS, int COLS>
__global__ __launch_bounds__(kThreads) void few_rows_kernel(const T* __restrict__ X, int N, int64_t ldx, const T* __restrict__ W,
                                                            int64_t ldw, int D, int M, int strips, Epilogue e) {
    constexpr int V = 16 / sizeof(T), LANES = COLS / V, STEP = kThreads / LANES, AHEAD = 4;
    __shared__ float part[kWaves][ROWS][COLS];
    const int strip = strip_of(blockIdx.x, strips);
    if (strip < 0) return;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int j = strip * COLS + lane % LANES * V;
    const bool whole = j + V <= M;
    float sum[ROWS][V] = {};
    const auto add = [&](auto count, int k0) {
        constexpr int n = decltype(count)::value;
        float w[n][V], x[n][ROWS];
#pragma unroll
        for (int a = 0; a < n; ++a) {
            const int64_t k = min(k0 + a * STEP, D - 1);  // past the last row: that one, and not added
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
    const int r = threadIdx.x / COLS, c = threadIdx.x % COLS, col = strip * COLS + c;
    if (r >= N || r >= ROWS || col >= M) return;
    float z[1][1] = {{0.f}}, bias[1];
#pragma unroll
    for (int w = 0; w < kWaves; ++w) z[0][0] += part[w][r][c];
    load_bias(e, col, M, bias);
    const int64_t row[1] = {r};
    finish<T>(e, row, col, N, M, bias, z);
}

typedef float f32x4 __attribute__((ext_vector_type(4)));

// A fragment of an operand, 16 outer indices from `first` on, one per lane, by the four k from `k` on.
template <bool K_INNER>
__device__ __forceinline__ void load_fragment(const PlainOperand& o, int64_t first, int64_t count, int64_t k, int64_t K, f32x4& v) {
    const float* const at = o.p + min(first + (threadIdx.x & 15), count - 1) * o.outer;
    if (K_INNER && k + 4 <= K) {
        float x[4];
        load_values(at + k, x);
        v = f32x4{x[0], x[1], x[2], x[3]};
    } else {
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const float x = at[min(k + r, K - 1) * o.inner];
            v[r] = k + r < K ? x : 0.f;
        }
    }
}

// 16 rows by 16 columns per workgroup on the fp32 matrix instructions, straight from memory: the wavefronts take every eighth 16 k,
// two of them ahead, and add up in LDS.  An instruction sums four k, one per 16 lanes: lane group q holds k = 4 q .. 4 q + 3 of both
// operands, and instruction r takes the r-th of each.  Blocks: row blocks * column blocks, row block fastest.  What bounds it is
// latency: 37 x 768 x 768 5.6 us, where the tiles of dense_tile_as_is.h take 7.4; from 128 rows on those are as fast.
struct PlainArgs {
    PlainOperand A, B;
    int64_t I, K;
    int J, row_blocks, col_blocks;
    Epilogue e;
};
struct PlainShared {
    float part[kWaves][16][17];
};
template <bool A_K, bool B_K>
__device__ __forceinline__ void plain_f32_block(const PlainArgs& args, int index, PlainShared& shared) {
    auto& part = shared.part;
    const PlainOperand &A = args.A, &B = args.B;
    const int64_t I = args.I, K = args.K;
    const int J = args.J, row_blocks = args.row_blocks;
    const Epilogue& e = args.e;
    const int block = strip_of(index, row_blocks * args.col_blocks);
    if (block < 0) return;
    const int64_t i0 = (int64_t)(block % row_blocks) * 16;
    const int j0 = block / row_blocks * 16;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, i16 = lane & 15, q = lane >> 4;
    f32x4 sum = {};
    struct Chunk {
        f32x4 a, b;
    };
    const auto load = [&](Chunk& c, int64_t k) {
        if (k >= K) return;
        load_fragment<B_K>(B, j0, J, k + 4 * q, K, c.b);
        load_fragment<A_K>(A, i0, I, k + 4 * q, K, c.a);
    };
    const auto multiply = [&](const Chunk& c) {
#pragma unroll
        for (int r = 0; r < 4; ++r) sum = __builtin_amdgcn_mfma_f32_16x16x4f32(c.b[r], c.a[r], sum, 0, 0, 0);
    };
    constexpr int STEP = 16 * kWaves;
    Chunk one, two;
    int64_t k = 16 * wave;
    load(one, k);
    load(two, k + STEP);
    for (; k < K; k += 2 * STEP) {
        {
            const Chunk now = one;
            load(one, k + 2 * STEP);
            multiply(now);
        }
        if (k + STEP >= K) break;
        const Chunk now = two;
        load(two, k + 3 * STEP);
        multiply(now);
    }
    // the first operand's index is the instruction's row: a lane has columns 4 q .. 4 q + 3 of row i16
#pragma unroll
    for (int r = 0; r < 4; ++r) part[wave][i16][4 * q + r] = sum[r];
    __syncthreads();
    const int v = threadIdx.x, col = j0 + v % 16;
    const int64_t row[1] = {i0 + v / 16};
    if (v >= 256 || row[0] >= I || col >= J) return;
    float z[1][1] = {{0.f}}, bias[1];
#pragma unroll
    for (int w = 0; w < kWaves; ++w) z[0][0] += part[w][v / 16][v % 16];
    load_bias(e, col, J, bias);
    finish<float>(e, row, col, I, J, bias, z);
}

template <bool A_K, bool B_K>
__global__ __launch_bounds__(kThreads) void plain_f32_kernel(PlainArgs a) {
    __shared__ PlainShared shared;
    plain_f32_block<A_K, B_K>(a, blockIdx.x, shared);
}

// Both gradients' products in one launch, and db's partial sums.
__global__ __launch_bounds__(kThreads) void plain_pair_kernel(PlainArgs x, PlainArgs w, int x_blocks, int w_blocks, PartialSums sums) {
    __shared__ __align__(8) PlainShared shared;
    const int b = blockIdx.x;
    if (b >= x_blocks + w_blocks)
        add_partial_sums<float, kThreads>(sums, b - x_blocks - w_blocks, &shared);
    else if (b < x_blocks)
        plain_f32_block<true, true>(x, b, shared);
    else
        plain_f32_block<false, false>(w, b - x_blocks, shared);
}

int64_t blocks_of(int64_t I, int J) { return ((I + 15) / 16) * ((J + 15) / 16); }

// Sets the blocks; how many workgroups they take, 0 for too many.
int count_blocks(PlainArgs& a) {
    const int64_t blocks = blocks_of(a.I, a.J);
    if (blocks > kMostTiles) return 0;
    a.row_blocks = (int)((a.I + 15) / 16), a.col_blocks = (a.J + 15) / 16;
    return (int)(blocks + 7) / 8 * 8;
}

// What a round of workgroups, one per compute unit, takes per k and beside that, in us: the three layouts' average over products of
// 8 x 768 x 768 to 128 x 768 x 2304.
constexpr float kLaunchUs = 2.6f, kPerK = 0.0033f, kRest = 0.27f;

}  // namespace

hipError_t launch_few_rows(int dtype, const void* X, int64_t N, int64_t ldx, const void* W, int64_t ldw, int D, int M,
                           const Epilogue& e, hipStream_t s) {
    // Wider strips read W in longer pieces, where there are enough of them: 1 x 8192 x 8192 in fp32 48 us by 16 columns, 41 by 32, 38 by
    // 64; 4096 wide 14, 13 and 19; in bf16 1 x 4096 x 11008 25, 21 and 32, 4096 wide 12, 16 and 29.  Long sums of few columns go by
    // strips of one load: 1 x 4096 x 1024 in fp32 10.5 us by 16 columns, 8.7 by four, in bf16 10.0 and 8.3 by eight; 1 x 768 x 768 3.9
    // and 3.9, in bf16 4.0 and 4.6.
    return with_type(dtype, [&](auto t) {
        using T = decltype(t);
        using std::integral_constant;
        constexpr int kEnough = 512 / sizeof(T), kLoad = 16 / sizeof(T);
        const auto launch = [&](auto rows, auto cols) {
            constexpr int ROWS = decltype(rows)::value, COLS = decltype(cols)::value;
            const int strips = (M + COLS - 1) / COLS;
            hipLaunchKernelGGL((few_rows_kernel<T, ROWS, COLS>), dim3((unsigned)(strips + 7) / 8 * 8), dim3(kThreads), 0, s,
                               static_cast<const T*>(X), (int)N, ldx, static_cast<const T*>(W), ldw, D, M, strips, e);
            return hipGetLastError();
        };
        const auto by_width = [&](auto rows) {
            if (D >= 2048 && M <= 256 * kLoad) return launch(rows, integral_constant<int, kLoad>());
            if constexpr (sizeof(T) == 4)
                if (M / 64 >= kEnough) return launch(rows, integral_constant<int, 64>());
            if (M / 32 >= kEnough) return launch(rows, integral_constant<int, 32>());
            return launch(rows, integral_constant<int, 16>());
        };
        if (N == 1) return by_width(integral_constant<int, 1>());
        if constexpr (sizeof(T) == 4) {
            if (N > 4) return by_width(integral_constant<int, 8>());
            if (N > 2) return by_width(integral_constant<int, 4>());
        }
        return by_width(integral_constant<int, 2>());
    });
}

hipError_t launch_plain_f32(const PlainOperand& A, const PlainOperand& B, int64_t I, int J, int64_t K, const Epilogue& e, hipStream_t s) {
    PlainArgs a = {A, B, I, K, J, 0, 0, e};
    const int blocks = count_blocks(a);
    if (blocks == 0) return hipErrorInvalidConfiguration;
    if (A.inner != 1)
        hipLaunchKernelGGL((plain_f32_kernel<false, false>), dim3(blocks), dim3(kThreads), 0, s, a);
    else if (B.inner == 1)
        hipLaunchKernelGGL((plain_f32_kernel<true, true>), dim3(blocks), dim3(kThreads), 0, s, a);
    else
        hipLaunchKernelGGL((plain_f32_kernel<true, false>), dim3(blocks), dim3(kThreads), 0, s, a);
    return hipGetLastError();
}

float plain_f32_us(int64_t I, int J, int64_t K) {
    const int64_t blocks = blocks_of(I, J);
    return blocks > kMostTiles ? 1e30f : kLaunchUs + std::ceil((float)blocks / compute_units()) * (K * kPerK + kRest);
}

hipError_t launch_plain_pair_f32(const float* dZ, int64_t ldg, const float* W, int64_t ldw, const float* X, int64_t ldx, int64_t N, int D,
                                 int M, const Epilogue& to_x, const Epilogue& to_w, const PartialSums& sums, hipStream_t s) {
    PlainArgs x = {{dZ, ldg, 1}, {W, ldw, 1}, N, M, D, 0, 0, to_x}, w = {{X, 1, ldx}, {dZ, 1, ldg}, D, N, M, 0, 0, to_w};
    const int x_blocks = count_blocks(x), w_blocks = count_blocks(w);
    if (x_blocks == 0 || w_blocks == 0) return hipErrorInvalidConfiguration;
    const unsigned blocks = x_blocks + w_blocks + (sums.out ? (sums.width + 31) / 32 : 0);
    hipLaunchKernelGGL(plain_pair_kernel, dim3(blocks), dim3(kThreads), 0, s, x, w, x_blocks, w_blocks, sums);
    return hipGetLastError();
}

// of workgroups of two kinds
float plain_pair_us(int64_t N, int D, int M) {
    const int64_t x_blocks = blocks_of(N, D), w_blocks = blocks_of(D, M);
    if (std::max(x_blocks, w_blocks) > kMostTiles) return 1e30f;
    const float x = M * kPerK + kRest, w = N * kPerK + kRest;
    return kLaunchUs + std::max(std::max(x, w), ((float)x_blocks * x + (float)w_blocks * w) / compute_units() + 1.4f * std::min(x, w));
}

}  // namespace lutnn
