// Dense layers of few rows: what bounds them is reading W once and the launch itself, so each is one launch that reads its operands
// as they are.
#include <algorithm>
#include <cmath>
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

// F fragments of an operand, 16 F outer indices from `first` on by 16 k: v[e][r] is the value at k + r, k being the lane group's first,
// and at the outer index that index_of(e, lane % 16) names: lanes read 16 bytes along k, or F neighbours at each k.
template <int F, bool K_INNER>
__device__ __forceinline__ int index_of(int e, int i) {
    return K_INNER ? 16 * e + i : F * i + e;
}
template <int F, bool K_INNER>
__device__ __forceinline__ void load_fragments(const PlainOperand& o, int64_t first, int64_t count, int64_t k, int64_t K, f32x4 (&v)[F]) {
    const int i = threadIdx.x & 15;
    if constexpr (K_INNER) {
#pragma unroll
        for (int e = 0; e < F; ++e) {
            const float* const at = o.p + min(first + 16 * e + i, count - 1) * o.outer;
            if (k + 4 <= K) {
                float x[4];
                load_values(at + k, x);
                v[e] = f32x4{x[0], x[1], x[2], x[3]};
            } else {
#pragma unroll
                for (int r = 0; r < 4; ++r) v[e][r] = k + r < K ? at[k + r] : 0.f;
            }
        }
    } else {
        const int64_t outer = first + F * i;
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const float* const at = o.p + min(k + r, K - 1) * o.inner;
            float x[F];
            if (outer + F <= count)
                load_values(at + outer, x);
            else
#pragma unroll
                for (int e = 0; e < F; ++e) x[e] = at[min(outer + e, count - 1)];
#pragma unroll
            for (int e = 0; e < F; ++e) v[e][r] = k + r < K ? x[e] : 0.f;
        }
    }
}

// 16 FI rows by 16 FJ columns per workgroup on the fp32 matrix instructions, straight from memory: the wavefronts take every eighth
// 16 k, two of them ahead, and add up in LDS.  An instruction sums four k, one per 16 lanes: lane group q holds k = 4 q .. 4 q + 3 of
// both operands, and instruction r takes the r-th of each.  Blocks: row blocks * column blocks, row block fastest.
struct PlainArgs {
    PlainOperand A, B;
    int64_t I, K;
    int J, row_blocks, col_blocks;
    Epilogue e;
};
template <int FI, int FJ>
struct PlainShared {
    float part[kWaves][FI * 16][16 * FJ + 1];
};
template <int FI, int FJ, bool A_K, bool B_K>
__device__ __forceinline__ void plain_f32_block(const PlainArgs& args, int index, PlainShared<FI, FJ>& shared) {
    constexpr int COLS = 16 * FJ;
    auto& part = shared.part;
    const PlainOperand &A = args.A, &B = args.B;
    const int64_t I = args.I, K = args.K;
    const int J = args.J, row_blocks = args.row_blocks;
    const Epilogue& e = args.e;
    const int block = strip_of(index, row_blocks * args.col_blocks);
    if (block < 0) return;
    const int64_t i0 = (int64_t)(block % row_blocks) * FI * 16;
    const int j0 = block / row_blocks * COLS;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, i16 = lane & 15, q = lane >> 4;
    f32x4 sum[FI][FJ] = {};
    struct Chunk {
        f32x4 a[FI], b[FJ];
    };
    const auto load = [&](Chunk& c, int64_t k) {
        if (k >= K) return;
        load_fragments<FJ, B_K>(B, j0, J, k + 4 * q, K, c.b);
        load_fragments<FI, A_K>(A, i0, I, k + 4 * q, K, c.a);
    };
    const auto multiply = [&](const Chunk& c) {
#pragma unroll
        for (int r = 0; r < 4; ++r)
#pragma unroll
            for (int i = 0; i < FI; ++i)
#pragma unroll
                for (int j = 0; j < FJ; ++j) sum[i][j] = __builtin_amdgcn_mfma_f32_16x16x4f32(c.b[j][r], c.a[i][r], sum[i][j], 0, 0, 0);
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
    for (int i = 0; i < FI; ++i)
#pragma unroll
        for (int j = 0; j < FJ; ++j)
#pragma unroll
            for (int r = 0; r < 4; ++r) part[wave][index_of<FI, A_K>(i, i16)][index_of<FJ, B_K>(j, 4 * q + r)] = sum[i][j][r];
    __syncthreads();
    for (int v = threadIdx.x; v < FI * 16 * COLS; v += kThreads) {
        const int64_t row[1] = {i0 + v / COLS};
        const int col = j0 + v % COLS;
        if (row[0] >= I || col >= J) continue;
        float z[1][1] = {{0.f}}, bias[1];
#pragma unroll
        for (int w = 0; w < kWaves; ++w) z[0][0] += part[w][v / COLS][v % COLS];
        load_bias(e, col, J, bias);
        finish<float>(e, row, col, I, J, bias, z);
    }
}

template <int FI, int FJ, bool A_K, bool B_K>
__global__ __launch_bounds__(kThreads) void plain_f32_kernel(PlainArgs a) {
    __shared__ PlainShared<FI, FJ> shared;
    plain_f32_block<FI, FJ, A_K, B_K>(a, blockIdx.x, shared);
}

// Both gradients' products in one launch, and db's partial sums.
template <int FI, int FJ>
__global__ __launch_bounds__(kThreads) void plain_pair_kernel(PlainArgs x, PlainArgs w, int x_blocks, int w_blocks, PartialSums sums) {
    __shared__ __align__(8) PlainShared<FI, FJ> shared;
    const int b = blockIdx.x;
    if (b >= x_blocks + w_blocks)
        add_partial_sums<kThreads>(sums, b - x_blocks - w_blocks, &shared);
    else if (b < x_blocks)
        plain_f32_block<FI, FJ, true, true>(x, b, shared);
    else
        plain_f32_block<FI, FJ, false, false>(w, b - x_blocks, shared);
}

// Fragments of rows and of columns per workgroup, and what a round of workgroups, one per compute unit, takes per k and beside that, in us: the three
// layouts' average over products of 37 x 768 to 2048 x 2048.  (Four by four spill.)
struct Block {
    int fi, fj;
    float per_k, rest;
};
constexpr Block kBlocks[] = {{1, 1, 0.0032f, 0.6f}, {2, 2, 0.0075f, 1.2f}, {4, 2, 0.0128f, 1.8f}};

float blocks_of(const Block& b, int64_t I, int J) {
    return (float)((I + 16 * b.fi - 1) / (16 * b.fi)) * (float)((J + 16 * b.fj - 1) / (16 * b.fj));
}

// A launch, and rounds of workgroups.
float block_us(const Block& b, int64_t I, int J, int64_t K, float units) {
    if (blocks_of(b, I, J) > kMostTiles) return 1e30f;
    return 3.f + std::ceil(blocks_of(b, I, J) / units) * (K * b.per_k + b.rest);
}

// ... of both gradients': of workgroups of two kinds
float pair_us(const Block& b, int64_t N, int D, int M, float units) {
    if (std::max(blocks_of(b, N, D), blocks_of(b, D, M)) > kMostTiles) return 1e30f;
    const float x = M * b.per_k + b.rest, w = N * b.per_k + b.rest;
    return 3.f + std::max(std::max(x, w), (blocks_of(b, N, D) * x + blocks_of(b, D, M) * w) / units + 0.5f * std::min(x, w));
}

template <class Us>
int best_block(Us&& us) {
    int best = 0;
    for (int i = 1; i < (int)(sizeof(kBlocks) / sizeof(kBlocks[0])); ++i)
        if (us(kBlocks[i]) < us(kBlocks[best])) best = i;
    return best;
}
int best_block(int64_t I, int J, int64_t K) {
    const float units = (float)compute_units();
    return best_block([&](const Block& b) { return block_us(b, I, J, K, units); });
}
int best_pair(int64_t N, int D, int M) {
    const float units = (float)compute_units();
    return best_block([&](const Block& b) { return pair_us(b, N, D, M, units); });
}

// Calls f with the fragments of a block.
template <class F>
hipError_t with_block(int block, F&& f) {
    using std::integral_constant;
    switch (block) {
        case 0: return f(integral_constant<int, 1>(), integral_constant<int, 1>());
        case 1: return f(integral_constant<int, 2>(), integral_constant<int, 2>());
        default: return f(integral_constant<int, 4>(), integral_constant<int, 2>());
    }
}

// Sets the blocks; how many workgroups they take, 0 for too many.
template <int FI, int FJ>
int count_blocks(PlainArgs& a) {
    const int64_t rows = (a.I + 16 * FI - 1) / (16 * FI), cols = (a.J + 16 * FJ - 1) / (16 * FJ);
    if (rows * cols > kMostTiles) return 0;
    a.row_blocks = (int)rows, a.col_blocks = (int)cols;
    return (int)(rows * cols + 7) / 8 * 8;
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
    return with_block(best_block(I, J, K), [&](auto fi, auto fj) {
        constexpr int FI = decltype(fi)::value, FJ = decltype(fj)::value;
        PlainArgs a = {A, B, I, K, J, 0, 0, e};
        const int blocks = count_blocks<FI, FJ>(a);
        if (blocks == 0) return hipErrorInvalidConfiguration;
        if (A.inner != 1)
            hipLaunchKernelGGL((plain_f32_kernel<FI, FJ, false, false>), dim3(blocks), dim3(kThreads), 0, s, a);
        else if (B.inner == 1)
            hipLaunchKernelGGL((plain_f32_kernel<FI, FJ, true, true>), dim3(blocks), dim3(kThreads), 0, s, a);
        else
            hipLaunchKernelGGL((plain_f32_kernel<FI, FJ, true, false>), dim3(blocks), dim3(kThreads), 0, s, a);
        return hipGetLastError();
    });
}

float plain_f32_us(int64_t I, int J, int64_t K) { return block_us(kBlocks[best_block(I, J, K)], I, J, K, (float)compute_units()); }

hipError_t launch_plain_pair_f32(const float* dZ, int64_t ldg, const float* W, int64_t ldw, const float* X, int64_t ldx, int64_t N, int D,
                                 int M, const Epilogue& to_x, const Epilogue& to_w, const PartialSums& sums, hipStream_t s) {
    return with_block(best_pair(N, D, M), [&](auto fi, auto fj) {
        constexpr int FI = decltype(fi)::value, FJ = decltype(fj)::value;
        PlainArgs x = {{dZ, ldg, 1}, {W, ldw, 1}, N, M, D, 0, 0, to_x}, w = {{X, 1, ldx}, {dZ, 1, ldg}, D, N, M, 0, 0, to_w};
        const int x_blocks = count_blocks<FI, FJ>(x), w_blocks = count_blocks<FI, FJ>(w);
        if (x_blocks == 0 || w_blocks == 0) return hipErrorInvalidConfiguration;
        const unsigned blocks = x_blocks + w_blocks + (sums.out ? (sums.width + 31) / 32 : 0);
        hipLaunchKernelGGL((plain_pair_kernel<FI, FJ>), dim3(blocks), dim3(kThreads), 0, s, x, w, x_blocks, w_blocks, sums);
        return hipGetLastError();
    });
}

float plain_pair_us(int64_t N, int D, int M) { return pair_us(kBlocks[best_pair(N, D, M)], N, D, M, (float)compute_units()); }

}  // namespace lutnn
