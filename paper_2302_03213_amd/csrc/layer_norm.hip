// Layer norm over the rows of a matrix, forward and backward: the normalisations between the linear layers of a model, whether
// those are looked up in tables or dense.
//
//   s = x + r          mu = sum s / D          rstd = 1 / sqrt(sum (s - mu)^2 / D + eps)          y = (s - mu) rstd w + b
//   h = (x - mu) rstd, q = g w:   dx = rstd (q - sum q / D - h sum (q h) / D) + r,   dw = sum_n g h,   db = sum_n g
//
// What bounds both: every matrix read or written once, at the rate of the memory.  A row lies in the registers of the threads
// that share it, 16 values each, so that nothing is read twice: the sum of squares is that of the differences from the mean (two
// reductions of a row, no cancellation).  Rows of up to 256 values take 16 threads, up to 1024 a wavefront, up to 4096 four, up
// to 8192 eight, up to 16384 sixteen.  Sums are fp32 ones.  16384 x 4096 in bf16 with a residual and its sum kept: 105 us, 537 MB
// at the rate of a large copy; a single row of 768 in fp32: 3.0, the latency of two loads and two reductions.
#include <algorithm>

#include "lutnn_kernels.h"
#include "matrix_types.h"

namespace lutnn {
namespace {

constexpr int kValues = 16;     // of a row, per thread
constexpr int kThreads = 256;   // per workgroup, but for rows that take more
constexpr int kMostBlocks = 1 << 21;  // a launch may have 2^32 threads

template <class T>
constexpr int kVector = 16 / sizeof(T);  // values per load

// A row's values as `TPR` threads hold them: vector c of thread t starts at column (c * TPR + t) * VEC.  The last vector of a row
// that is no whole number of them is moved back to end with it; what it then repeats of its neighbour's counts as zero in sums
// and is stored twice, with the same value.
template <int VEC, int TPR>
struct Columns {
    int D, t;
    __device__ __forceinline__ int start(int c) const { return (c * TPR + t) * VEC; }
    __device__ __forceinline__ bool any(int c) const { return start(c) < D; }
    __device__ __forceinline__ int at(int c) const { return min(start(c), D - VEC); }
    __device__ __forceinline__ bool mine(int c, int j) const { return at(c) + j >= start(c); }
};

// The sums over a row's threads, in every one of them.  shared: 2 * count floats per wavefront, the halves in turn.
template <int TPR, int count>
__device__ __forceinline__ void row_sums(float (&v)[count], float* shared, int& turn) {
#pragma unroll
    for (int d = 1; d < (TPR < 64 ? TPR : 64); d *= 2)
#pragma unroll
        for (int i = 0; i < count; ++i) v[i] += __shfl_xor(v[i], d, 64);
    if constexpr (TPR > 64) {
        constexpr int kWaves = TPR / 64;
        float* const slot = shared + turn * count * kWaves;
        turn ^= 1;
        if ((threadIdx.x & 63) == 0)
#pragma unroll
            for (int i = 0; i < count; ++i) slot[i * kWaves + (threadIdx.x >> 6)] = v[i];
        __syncthreads();  // one is enough: a half is written again only behind the other half's barrier
#pragma unroll
        for (int i = 0; i < count; ++i) {
            v[i] = 0.f;
#pragma unroll
            for (int w = 0; w < kWaves; ++w) v[i] += slot[i * kWaves + w];
        }
    }
}

template <class T>
struct NormArgs {
    const T *X, *R;
    const float *w, *b;
    T *Y, *S;
    float* statistics;
    int64_t N, ldx, ldr, ldy, lds;
    int D;
    float eps;
};

// kThreads / TPR rows (or one) per workgroup, the first ones and then every grid's worth further.
template <class T, int VEC, int TPR>
__global__ __launch_bounds__(TPR < kThreads ? kThreads : TPR) void layer_norm_kernel(NormArgs<T> a) {
    constexpr int ROWS = TPR < kThreads ? kThreads / TPR : 1, CH = VEC == 1 ? 1 : kValues / VEC;
    __shared__ float shared[2 * (TPR > 64 ? TPR / 64 : 1)];
    int turn = 0;
    const Columns<VEC, TPR> col{a.D, (int)(threadIdx.x % TPR)};
    // rows that end earlier than a workgroup's others are whole wavefronts' or, in groups of 16, nobody that those wait for
    for (int64_t n = (int64_t)blockIdx.x * ROWS + threadIdx.x / TPR; n < a.N; n += (int64_t)gridDim.x * ROWS) {
        float x[CH][VEC], total[1] = {0.f};
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            if (!col.any(c)) continue;
            load_values(a.X + n * a.ldx + col.at(c), x[c]);
            if (a.R) {
                float r[VEC];
                load_values(a.R + n * a.ldr + col.at(c), r);
#pragma unroll
                for (int j = 0; j < VEC; ++j) x[c][j] += r[j];
                if (a.S) store_values(a.S + n * a.lds + col.at(c), x[c]);
            }
#pragma unroll
            for (int j = 0; j < VEC; ++j) total[0] += col.mine(c, j) ? x[c][j] : 0.f;
        }
        row_sums<TPR>(total, shared, turn);
        const float mean = total[0] / a.D;
        float squares[1] = {0.f};
#pragma unroll
        for (int c = 0; c < CH; ++c)
            if (col.any(c))
#pragma unroll
                for (int j = 0; j < VEC; ++j) {
                    x[c][j] -= mean;
                    squares[0] += col.mine(c, j) ? x[c][j] * x[c][j] : 0.f;
                }
        row_sums<TPR>(squares, shared, turn);
        const float rstd = 1.f / sqrtf(squares[0] / a.D + a.eps);
        if (a.statistics && col.t == 0) {
            a.statistics[2 * n] = mean;
            a.statistics[2 * n + 1] = rstd;
        }
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            if (!col.any(c)) continue;
#pragma unroll
            for (int j = 0; j < VEC; ++j) x[c][j] *= rstd;
            if (a.w) {
                float w[VEC];
                load_values(a.w + col.at(c), w);
#pragma unroll
                for (int j = 0; j < VEC; ++j) x[c][j] *= w[j];
            }
            if (a.b) {
                float b[VEC];
                load_values(a.b + col.at(c), b);
#pragma unroll
                for (int j = 0; j < VEC; ++j) x[c][j] += b[j];
            }
            store_values(a.Y + n * a.ldy + col.at(c), x[c]);
        }
    }
}

template <class T>
struct NormGradientArgs {
    const T *G, *X, *R;
    const float *statistics, *w;
    T* dX;
    float* partial;  // [workgroups][2][D]
    int64_t N, ldg, ldx, ldr, lddx;
    int D, row_blocks;
    float *dw, *db;  // of the workgroups behind row_blocks
};

// dw and db of THREADS / 16 columns, every row of them read again, by 16 groups of threads.  part: two per thread.  A thread adds up
// 64 rows, in 64 bits: as an fp32 chain they were 1.5 times as far off as a plain sum by trees.  1024 x 768 6.2 us for 6.0 so, in
// bf16 6.1 for 5.9, 1024 x 4096 22.9 for 22.8, in bf16 14.9 for 14.8.
template <class T, int THREADS>
__device__ __forceinline__ void sum_columns(const NormGradientArgs<T>& a, int block, double* part) {
    constexpr int GROUPS = 16, COLUMNS = THREADS / GROUPS;
    const int group = threadIdx.x / COLUMNS, d = block * COLUMNS + threadIdx.x % COLUMNS, at = min(d, a.D - 1);
    double sums[2] = {0, 0};
#pragma unroll 8
    for (int64_t n = group; n < a.N; n += GROUPS) {
        const float g = (float)a.G[n * a.ldg + at], x = (float)a.X[n * a.ldx + at];
        sums[0] = __fma_rn((double)g, (double)((x - a.statistics[2 * n]) * a.statistics[2 * n + 1]), sums[0]);
        sums[1] += g;
    }
    part[2 * threadIdx.x] = sums[0];
    part[2 * threadIdx.x + 1] = sums[1];
    __syncthreads();
    if (group != 0 || d >= a.D) return;
#pragma unroll
    for (int i = 1; i < GROUPS; ++i)
#pragma unroll
        for (int v = 0; v < 2; ++v) sums[v] += part[2 * (threadIdx.x + i * COLUMNS) + v];
    if (a.dw) a.dw[d] = (float)sums[0];
    if (a.db) a.db[d] = (float)sums[1];
}

// Rows are dealt to the workgroups in turn; each keeps the column sums of its own in registers and leaves them in `partial`.  The fewer
// workgroups, the fewer sums are left, so that the next row's loads have to hide the memory's latency: 16384 x 4096 in bf16 with a
// residual 107 us, 537 MB at the rate of a large copy; 168 without them.  SUMS: whether any are kept.
template <class T, int VEC, int TPR, bool SUMS>
__global__ __launch_bounds__(TPR < kThreads ? kThreads : TPR) void layer_norm_gradient_kernel(NormGradientArgs<T> a) {
    constexpr int THREADS = TPR < kThreads ? kThreads : TPR, ROWS = THREADS / TPR, CH = VEC == 1 ? 1 : kValues / VEC;
    __shared__ float shared[4 * (TPR > 64 ? TPR / 64 : 1)];
    constexpr bool PARTS = SUMS && ROWS > 1;
    __shared__ float parts[2][PARTS ? CH * VEC : 1][PARTS ? THREADS : 1];
    __shared__ double columns[SUMS ? 1 : 2 * THREADS];
    if (!SUMS && (int)blockIdx.x >= a.row_blocks) return sum_columns<T, THREADS>(a, blockIdx.x - a.row_blocks, columns);
    int turn = 0;
    const Columns<VEC, TPR> col{a.D, (int)(threadIdx.x % TPR)};
    float dw[CH][VEC] = {}, db[CH][VEC] = {}, w[CH][VEC];
    const auto load_weight = [&] {
#pragma unroll
        for (int c = 0; c < CH; ++c)
            if (col.any(c)) {
                if (a.w)
                    load_values(a.w + col.at(c), w[c]);
                else
#pragma unroll
                    for (int j = 0; j < VEC; ++j) w[c][j] = 1.f;
            }
    };
    // a row as it lies in memory; the next one is on its way while one is worked on, where there are registers for it: sixteen
    // wavefronts have 128 each
    constexpr bool AHEAD = TPR < 1024;
    struct Row {
        typename Packed<T, VEC>::type g[CH], x[CH], r[CH];
        float mean, rstd;
    };
    const auto fetch = [&](Row& row, int64_t n) {
        if (n >= a.N) return;
        row.mean = a.statistics[2 * n];
        row.rstd = a.statistics[2 * n + 1];
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            if (!col.any(c)) continue;
            row.g[c] = *reinterpret_cast<const typename Packed<T, VEC>::type*>(a.G + n * a.ldg + col.at(c));
            row.x[c] = *reinterpret_cast<const typename Packed<T, VEC>::type*>(a.X + n * a.ldx + col.at(c));
            if (a.R && a.dX) row.r[c] = *reinterpret_cast<const typename Packed<T, VEC>::type*>(a.R + n * a.ldr + col.at(c));
        }
    };
    const auto value = [](const typename Packed<T, VEC>::type& v, int j) {
        if constexpr (VEC == 1)
            return (float)v;
        else
            return (float)v[j];
    };
    const int64_t first = (int64_t)blockIdx.x * ROWS + threadIdx.x / TPR, step = (int64_t)a.row_blocks * ROWS;
    Row next;
    if constexpr (AHEAD) {
        load_weight();
        fetch(next, first);
    }
    for (int64_t n = first; n < a.N; n += step) {
        if constexpr (!AHEAD) fetch(next, n);
        const Row row = next;
        if constexpr (AHEAD)
            fetch(next, n + step);
        else
            load_weight();
        float g[CH][VEC], h[CH][VEC], sums[2] = {0.f, 0.f};
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            if (!col.any(c)) continue;
#pragma unroll
            for (int j = 0; j < VEC; ++j) {
                g[c][j] = value(row.g[c], j);
                h[c][j] = (value(row.x[c], j) - row.mean) * row.rstd;
                if (SUMS && col.mine(c, j)) {
                    dw[c][j] = __fmaf_rn(g[c][j], h[c][j], dw[c][j]);
                    db[c][j] += g[c][j];
                }
                g[c][j] *= w[c][j];
                sums[0] += col.mine(c, j) ? g[c][j] : 0.f;
                sums[1] += col.mine(c, j) ? g[c][j] * h[c][j] : 0.f;
            }
        }
        if (SUMS && !a.dX) continue;
        row_sums<TPR>(sums, shared, turn);
        const float q = sums[0] / a.D, qh = sums[1] / a.D;
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            if (!col.any(c)) continue;
#pragma unroll
            for (int j = 0; j < VEC; ++j) {
                g[c][j] = row.rstd * (g[c][j] - q - h[c][j] * qh);
                if (a.R) g[c][j] += value(row.r[c], j);
            }
            store_values(a.dX + n * a.lddx + col.at(c), g[c]);
        }
    }
    if constexpr (!SUMS) return;
    float* const mine = a.partial + (int64_t)blockIdx.x * 2 * a.D;
    if constexpr (ROWS > 1) {  // the workgroup's rows, in order, a column per thread and turn
#pragma unroll
        for (int c = 0; c < CH; ++c)
#pragma unroll
            for (int j = 0; j < VEC; ++j) {
                parts[0][c * VEC + j][threadIdx.x] = dw[c][j];
                parts[1][c * VEC + j][threadIdx.x] = db[c][j];
            }
        __syncthreads();
        for (int v = threadIdx.x; v < CH * VEC * TPR; v += THREADS) {
            const int value = v / TPR, t = v % TPR, c = value / VEC, j = value % VEC;
            const Columns<VEC, TPR> of{a.D, t};
            if (!of.any(c) || !of.mine(c, j)) continue;
            float sums[2] = {0.f, 0.f};
#pragma unroll
            for (int r = 0; r < ROWS; ++r)
#pragma unroll
                for (int i = 0; i < 2; ++i) sums[i] += parts[i][value][r * TPR + t];
            mine[of.at(c) + j] = sums[0];
            mine[a.D + of.at(c) + j] = sums[1];
        }
    } else {
#pragma unroll
        for (int c = 0; c < CH; ++c)
            if (col.any(c))
#pragma unroll
                for (int j = 0; j < VEC; ++j)
                    if (col.mine(c, j)) {
                        mine[col.at(c) + j] = dw[c][j];
                        mine[a.D + col.at(c) + j] = db[c][j];
                    }
    }
}

template <class T, class F>
hipError_t by_width(int D, F&& f) {
    using std::integral_constant;
    constexpr int V = kVector<T>;
    if (D < V) return f(integral_constant<int, 1>(), integral_constant<int, 16>());
    if (D <= 16 * kValues) return f(integral_constant<int, V>(), integral_constant<int, 16>());
    if (D <= 64 * kValues) return f(integral_constant<int, V>(), integral_constant<int, 64>());
    if (D <= 256 * kValues) return f(integral_constant<int, V>(), integral_constant<int, 256>());
    if (D <= 512 * kValues) return f(integral_constant<int, V>(), integral_constant<int, 512>());
    return f(integral_constant<int, V>(), integral_constant<int, 1024>());
}

int rows_per_workgroup(int D) { return D <= 16 * kValues ? kThreads / 16 : D <= 64 * kValues ? kThreads / 64 : 1; }

// Few rows are read again for dw and db beside dX, and not summed by workgroup and then over those.  us so and the other way, by rows:
//   fp32   1024 x 1032 11.0, 12.0;  896 x 2048 12.0, 13.5;  1024 x 2048 13.8, 13.8 (with a residual 17.1, 13.9);  768 x 3000 14.0, 15.1;
//          896 x 3000 17.1, 16.3;  768 x 4096 16.2, 16.5;  1024 x 4096 23.3, 18.9;  1024 x 5120 19.8, 19.8;  1024 x 16384 68, 94
//   bf16   1024 x 1032 7.7, 11.9;  1024 x 2048 10.1, 13.8;  1024 x 4096 15.2, 20.5;  1024 x 5120 13.9, 21.4;  1024 x 16384 33, 57
// Above 4096 values a workgroup has more threads, and takes more columns.  From 1025 rows on both ways are near each other at most
// widths: 1536 x 1024 12.9, 10.6 (bf16 10.2, 10.7), 1536 x 4096 32, 21 (21, 21), 1536 x 8192 38, 33 (27, 30).
int64_t direct_rows(int dtype, int D) { return dtype == 0 && D > 2048 && D <= 256 * kValues ? 768 : 1024; }

// Two workgroups per compute unit; one for rows of more than four wavefronts, and, where sums are left (row_bytes: what a row reads
// then), where the memory is what they wait for, and for few rows beside wide sums.  us by one and by two:
//   6 KB (bf16, 1024 wide, a residual)  4096 rows 12.4, 13.4;  16384 28.7, 27.1       12 KB (fp32, 1536)  4096 26.4, 20.2;  16384 84, 62
//   16 KB (bf16, 4096)  4096 35.9, 33.4;  16384 106, 86                               23.5 KB (fp32, 3008)  8192 55.3, 53.0;  16384 107, 116
//   24 KB (bf16, 4096, a residual)  4096 37.2, 36.6;  8192 60.9, 54.0;  16384 109, 110
//         (fp32, 2048, a residual)  4096 28.6, 27.7;  8192 48.6, 45.2;  16384 95.9, 101.6
//   28 KB (fp32, 3584)  4096 35.2, 35.6;  16384 136, 140          30 KB (fp32, 2560, a residual)  4096 31.8, 32.6;  16384 125, 133
//   48 KB (fp32, 4096, a residual)  4096 47.1, 49.0;  16384 199, 209
// so at 24 KB it is one where G, X and the residual pass the 256 MB cache.  Few rows: 2048 x 3008 in bf16 21.6, 22.2, 2048 x 4096 24.0,
// 26.8 (fp32 24.5, 26.2), 1100 x 2560 16.5, 19.1, but 2048 x 2560 in fp32 20.0, 19.1, and 3080 x 4096 30.6, 29.8.
int gradient_workgroups(int64_t N, int D, int sums, int64_t row_bytes = 0) {
    const bool busy = row_bytes > 24 << 10 || (row_bytes == 24 << 10 && N * row_bytes > 256 << 20);
    const bool one = sums > 0 ? sums == 1 : D > 256 * kValues || busy || (row_bytes > 0 && N <= 2048 && D > 2048);
    const int64_t most = (one ? 1 : 2) * (int64_t)compute_units();
    const int rows = rows_per_workgroup(D);
    return (int)std::min<int64_t>((N + rows - 1) / rows, most);
}

bool direct_sums(int dtype, int64_t N, int D, int sums) { return sums >= 0 ? sums == 0 : N <= direct_rows(dtype, D); }

}  // namespace

size_t layer_norm_gradient_workspace(int dtype, int64_t N, int D, int sums) {
    return direct_sums(dtype, N, D, sums) ? 0 : (size_t)gradient_workgroups(N, D, sums) * 2 * D * sizeof(float);
}

hipError_t launch_layer_norm(int dtype, const void* X, int64_t N, int64_t ldx, int D, const void* R, int64_t ldr, const float* w,
                             const float* b, float eps, void* Y, int64_t ldy, void* S, int64_t lds, float* statistics,
                             hipStream_t s) {
    return with_type(dtype, [&](auto t) {
        using T = decltype(t);
        const NormArgs<T> a{static_cast<const T*>(X), static_cast<const T*>(R), w, b, static_cast<T*>(Y), static_cast<T*>(S),
                            statistics, N, ldx, ldr, ldy, lds, D, eps};
        return by_width<T>(D, [&](auto vec, auto tpr) {
            constexpr int TPR = decltype(tpr)::value, ROWS = TPR < kThreads ? kThreads / TPR : 1;
            hipLaunchKernelGGL((layer_norm_kernel<T, decltype(vec)::value, TPR>), dim3((unsigned)std::min<int64_t>((N + ROWS - 1) / ROWS, kMostBlocks)),
                               dim3(TPR < kThreads ? kThreads : TPR), 0, s, a);
            return hipGetLastError();
        });
    });
}

hipError_t launch_layer_norm_gradient(int dtype, const void* G, int64_t N, int64_t ldg, const void* X, int64_t ldx, int D,
                                      const float* statistics, const float* w, const void* R, int64_t ldr, void* dX, int64_t lddx,
                                      float* dw, float* db, int sums, void* workspace, hipStream_t s) {
    const bool direct = direct_sums(dtype, N, D, sums) && (dw || db);
    float* const partial = !direct && (dw || db) ? static_cast<float*>(workspace) : nullptr;
    const int64_t row_bytes = partial ? (int64_t)D * (dtype == 0 ? 4 : 2) * (R && dX ? 3 : 2) : 0;
    const int groups = gradient_workgroups(N, D, sums, row_bytes), rows = dX || partial ? groups : 0;
    if (groups > 0) {
        const hipError_t e = with_type(dtype, [&](auto t) {
            using T = decltype(t);
            const NormGradientArgs<T> a{static_cast<const T*>(G), static_cast<const T*>(X), static_cast<const T*>(R), statistics, w,
                                        static_cast<T*>(dX), partial, N, ldg, ldx, ldr, lddx, D, rows, dw, db};
            return by_width<T>(D, [&](auto vec, auto tpr) {
                constexpr int TPR = decltype(tpr)::value;
                constexpr int THREADS = TPR < kThreads ? kThreads : TPR, COLUMNS = THREADS / 16;
                const dim3 grid((unsigned)(rows + (direct ? (D + COLUMNS - 1) / COLUMNS : 0))), threads(THREADS);
                if (partial)
                    hipLaunchKernelGGL((layer_norm_gradient_kernel<T, decltype(vec)::value, TPR, true>), grid, threads, 0, s, a);
                else
                    hipLaunchKernelGGL((layer_norm_gradient_kernel<T, decltype(vec)::value, TPR, false>), grid, threads, 0, s, a);
                return hipGetLastError();
            });
        });
        if (e != hipSuccess) return e;
    }
    if ((!dw && !db) || (direct && N > 0)) return hipSuccess;
    return launch_partial_sums(partial, groups, 2 * D, D, dw, db, s);
}

}  // namespace lutnn
