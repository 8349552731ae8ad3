// Linear layers that are not looked up: Y = act(X W + b) + R, and the gradients of X, W and b.
//
//   Z = X W + b,  Y = act(Z) + R;      dZ = dL/dY act'(Z),  dX = dZ W^T,  dW = X^T dZ,  db = sum over rows of dZ
//
// The three products run on the matrix cores (dense_product.h), which want 16-bit operands whose rows are whole aligned 16-byte
// vectors.  Matrices that are such go to them as they are; others are laid out in the workspace first: fp32 ones as three planes of
// bf16 parts, 16-bit ones of odd widths, strides or addresses as copies with padded rows.  dZ is formed on the way there, and summed
// for db in the same pass: 8192 x 4096 in bf16 with the slope of gelu_tanh 44 us, 4.6 TB/s.  Products too small for that take
// their operands as they are (dense_tile_as_is.h; dense_rows.hip: fp32 ones of up to a hundred rows, a few rows of any type).
#include <algorithm>
#include <cmath>
#include <type_traits>

#include "dense_product.h"
#include "dense_rows.h"

namespace lutnn {
namespace {

constexpr int kVec = 8;                      // columns per thread of the passes over a matrix
constexpr int64_t kDirectRows = 2048;        // of a bias' gradient that has no pass of its own
constexpr int64_t kMaxStride = 1 << 21;      // values: a tile's rows within 32-bit offsets

int64_t round_up(int64_t v, int64_t to) { return (v + to - 1) / to * to; }

bool usable(int dtype, const void* p, int64_t ld, int64_t width) {
    return dtype != 0 && (reinterpret_cast<uintptr_t>(p) & 15) == 0 && ld % 8 == 0 && width % 8 == 0 && ld <= kMaxStride;
}

int64_t laid_out_stride(int64_t width) { return round_up(width, 8); }
size_t laid_out_bytes(int dtype, int64_t rows, int64_t width) {
    return (size_t)round_up((dtype == 0 ? 3 : 1) * rows * laid_out_stride(width) * 2, 256);
}

// in kernels
__device__ __forceinline__ int64_t round8(int64_t width) { return (width + 7) / 8 * 8; }
__device__ __forceinline__ int64_t laid_out_units(int64_t width) { return (width + kVec - 1) / kVec; }

// Eight values of a row, those past its end as zeros.
template <class T>
__device__ __forceinline__ void load_row(const T* row, int64_t col, int64_t width, float (&v)[kVec]) {
    if (col + kVec <= width) {
        load_values(row + col, v);
        return;
    }
#pragma unroll
    for (int i = 0; i < kVec; ++i) v[i] = col + i < width ? (float)row[col + i] : 0.f;
}

// Eight values to where the matrix cores read them: fp32 ones as their parts.
template <class T>
__device__ __forceinline__ void lay_out(const float (&v)[kVec], uint16_t* to, int64_t plane) {
    if constexpr (sizeof(T) == 4) {
        typedef unsigned u32x4 __attribute__((ext_vector_type(4)));
        uint32_t bits[kVec], high[4], mid[4], low[4];
#pragma unroll
        for (int i = 0; i < kVec; ++i) bits[i] = __float_as_uint(v[i]);
        cut<4>(bits, high, mid, low);
        *reinterpret_cast<u32x4*>(to) = u32x4{high[0], high[1], high[2], high[3]};
        *reinterpret_cast<u32x4*>(to + plane) = u32x4{mid[0], mid[1], mid[2], mid[3]};
        *reinterpret_cast<u32x4*>(to + 2 * plane) = u32x4{low[0], low[1], low[2], low[3]};
    } else {
        store_values(reinterpret_cast<T*>(to), v);
    }
}

// Up to two matrices laid out in one launch.
struct LayOut {
    const void* from[2];
    int64_t ld[2], rows[2], width[2];
    uint16_t* to[2];
};

// By workgroup `block` of `blocks` of 256 threads.
template <class T>
__device__ __forceinline__ void lay_out_matrices(const LayOut& a, int block, int blocks) {
    int64_t units[2];
    for (int m = 0; m < 2; ++m) units[m] = a.to[m] ? a.rows[m] * (laid_out_units(a.width[m])) : 0;
    for (int64_t v = block * 256LL + threadIdx.x; v < units[0] + units[1]; v += blocks * 256LL) {
        const int m = v >= units[0];
        const int64_t u = m ? v - units[0] : v, per_row = laid_out_units(a.width[m]);
        const int64_t row = u / per_row, col = (u - row * per_row) * kVec;
        float x[kVec];
        load_row(static_cast<const T*>(a.from[m]) + row * a.ld[m], col, a.width[m], x);
        lay_out<T>(x, a.to[m] + u * kVec, a.rows[m] * per_row * kVec);
    }
}

template <class T>
__global__ __launch_bounds__(256) void lay_out_kernel(LayOut a) {
    lay_out_matrices<T>(a, blockIdx.x, gridDim.x);
}

struct SlopeArgs {
    const void *G, *Z;
    int64_t ldg, ldz, N;
    int M, activation;
    uint16_t* to;    // dZ laid out; may be missing
    bool plain;      // ... or, of fp32, as it is
    float* partial;  // [row chunks][M] sums of dZ's columns; may be missing
    int lanes, col_tiles, chunks;
};

// dZ = G act'(Z), laid out, and its column sums.  A workgroup takes 8 * lanes columns and every chunks-th group of rows; a thread
// keeps its eight columns.  grid: chunks * col_tiles, column tile fastest; those behind them lay X and W out.
// Of 16-bit matrices dZ is rounded to their type, as the matrix instructions multiply no other.  G alone needs no rounding and relu's
// slope none either; any other slope costs dX and dW as much again as their own rounding, in the 2-norm 1.66e-3 -> 2.35e-3 in bf16 and
// 2.1e-4 -> 2.9e-4 in fp16.  In two parts, dZ as exact as fp32, every sum is twice as long: dX and dW of 8192 x 4096 x 4096 in bf16
// 208 + 201 us by themselves, 395 + 401 so.  Not taken: an optimizer's step sees the gradients' own rounding either way.
template <class T>
__global__ __launch_bounds__(256) void slope_kernel(SlopeArgs a, LayOut others) {
    __shared__ float part[256][kVec + 1];
    const int own = a.chunks * a.col_tiles;
    if ((int)blockIdx.x >= own) return lay_out_matrices<T>(others, blockIdx.x - own, gridDim.x - own);
    const int sub = threadIdx.x / a.lanes, lane = threadIdx.x % a.lanes, rows = 256 / a.lanes;
    const int64_t col = ((int64_t)(blockIdx.x % a.col_tiles) * a.lanes + lane) * kVec;
    const int chunk = blockIdx.x / a.col_tiles;
    const int64_t ldt = round8(a.M);
    float sum[kVec] = {};
    if (col < a.M) {
        for (int64_t n = (int64_t)chunk * rows + sub; n < a.N; n += (int64_t)a.chunks * rows) {
            float g[kVec];
            load_row(static_cast<const T*>(a.G) + n * a.ldg, col, a.M, g);
            if (a.activation) {
                float z[kVec];
                load_row(static_cast<const T*>(a.Z) + n * a.ldz, col, a.M, z);
                slope_all(g, z, a.activation);
            }
#pragma unroll
            for (int i = 0; i < kVec; ++i) sum[i] += g[i];
            if (a.to && a.plain) {
                float* const at = reinterpret_cast<float*>(a.to) + n * a.M + col;
#pragma unroll
                for (int i = 0; i < kVec; ++i)
                    if (col + i < a.M) at[i] = g[i];
            } else if (a.to) {
                lay_out<T>(g, a.to + n * ldt + col, a.N * ldt);
            }
        }
    }
    if (!a.partial) return;
#pragma unroll
    for (int i = 0; i < kVec; ++i) part[threadIdx.x][i] = sum[i];
    __syncthreads();
    for (int v = threadIdx.x; v < a.lanes * kVec; v += 256) {
        const int64_t m = (int64_t)(blockIdx.x % a.col_tiles) * a.lanes * kVec + v;
        float total = 0.f;
        for (int r = 0; r < rows; ++r) total += part[r * a.lanes + v / kVec][v % kVec];
        if (m < a.M) a.partial[(int64_t)chunk * a.M + m] = total;
    }
}

// How the rows are shared out: a power of two of lanes per row, and eight rows per thread or 4 workgroups per compute unit.
void share_rows(int64_t N, int M, SlopeArgs& a) {
    a.lanes = 1;
    while (a.lanes < 64 && a.lanes * kVec < M) a.lanes *= 2;
    a.col_tiles = (int)((M + a.lanes * kVec - 1) / (a.lanes * kVec));
    const int64_t per_chunk = 256 / a.lanes * 8;
    a.chunks = (int)std::max<int64_t>(1, std::min<int64_t>((N + per_chunk - 1) / per_chunk, std::max(4 * compute_units() / a.col_tiles, 1)));
}

// dW and db of no rows
template <class T>
__global__ __launch_bounds__(256) void clear_kernel(T* dW, int64_t ld, int64_t rows, int M, float* db) {
    for (int64_t v = blockIdx.x * 256LL + threadIdx.x; v < (rows + 1) * M; v += gridDim.x * 256LL) {
        const int64_t row = v / M, m = v - row * M;
        if (row < rows) {
            if (dW) dW[row * ld + m] = (T)0.f;
        } else if (db) {
            db[m] = 0.f;
        }
    }
}

hipError_t launch_clear(int dtype, void* dW, int64_t ld, int D, int M, float* db, hipStream_t s) {
    if (!dW && !db) return hipSuccess;
    return with_type(dtype, [&](auto t) {
        using T = decltype(t);
        hipLaunchKernelGGL(clear_kernel<T>, dim3(1024), dim3(256), 0, s, static_cast<T*>(dW), ld, (int64_t)D, M, db);
        return hipGetLastError();
    });
}

// The tiles of with_tile (dense_product.h), how many of them a compute unit holds, and what 1 .. that many at once take, in us: per
// 64 k, and beside that.  16 bits: from products of 16 x 16 n tiles at K = 512 and 2560, the three layouts' average.  Small tiles are
// bound by what a compute unit gets from L2 (75 GB/s), the large ones by the matrix instructions and the power they draw.  fp32: fitted
// to the times of 28 sizes from 8 x 768 x 768 to 4096 x 4096 x 768, three products each, which they then order so that the choice
// takes 2 % longer than the best of all; tiles of 64 x 64 and 64 x 128 from planes were the best of none by more than 1 %.  At 56 sizes
// that nothing was fitted to, 24 to 6000 rows by widths of 512 to 4608, the choice takes 3 % longer than the best tile (forward, both
// gradients and dW alone; at worst 40 %, both gradients of 24 x 640 x 2560), in bf16 1, 4 and 2 % (69 %, those of 24 x 4608 x 1152).
struct TileSize {
    int i, j, depth, at_once;
    float stage[4], rest[4];
    bool as_is = false;  // of operands that are not laid out
};
constexpr TileSize kTiles16[] = {{256, 256, 32, 1, {1.55f}, {9.0f}},
                                 {128, 128, 64, 2, {0.78f, 0.90f}, {2.0f, 5.0f}},
                                 {64, 128, 64, 2, {0.61f, 0.65f}, {0.5f, 2.5f}},
                                 {64, 64, 64, 3, {0.23f, 0.46f, 0.66f}, {1.0f, 0.7f, 1.0f}},
                                 {32, 64, 64, 4, {0.16f, 0.37f, 0.56f, 0.72f}, {1.0f, 0.5f, 0.5f, 0.5f}},
                                 {64, 64, 64, 2, {0.42f, 0.85f}, {1.4f, 1.8f}, true},
                                 {32, 64, 64, 4, {0.37f, 0.60f, 0.75f, 1.10f}, {0.6f, 0.9f, 0.9f, 1.0f}, true}};
constexpr TileSize kTilesF32[] = {{128, 256, 32, 1, {3.3f}, {8.4f}},
                                  {128, 128, 32, 1, {2.02f}, {3.7f}},
                                  {64, 64, 32, 2, {1.08f, 2.07f}, {1.5f, 1.7f}, true},
                                  {32, 32, 32, 2, {0.32f, 0.56f}, {0.8f, 0.8f}, true}};
constexpr float kLaunchUs = 3.5f, kNever = 1e30f;

// What sharing a sum out costs beside the shares: the second launch, and the shares written and read again.  One 16-bit product's are set
// by what they choose, not timed by themselves: 64 x 4096 x 4096 in bf16 13.3 us by four, 17.1 by tiles of half the rows, as kJoin has
// it; both gradients' products chosen by kJoin16 took up to 14 % longer.
struct Join {
    float us, bytes_per_us;
};
constexpr Join kJoin = {5.f, 3.5e6f}, kJoin16 = {3.5f, 5e6f};

// Laying that many values out: fp32 ones read, and written as three parts, much of both in the caches; 16-bit ones from rows of any
// alignment, none of them nothing.
float lay_out_us(int dtype, float values) {
    if (dtype == 0) return 2.5f + values * 10 / 10e6f;
    return values > 0.f ? 2.7f + values * 4 / 2.6e6f : 0.f;
}

// A product's tile, how many of its tiles are one workgroup's, and how many workgroups share the sum of each of the others.
struct Plan {
    int tile, whole, splits;
    int64_t tiles;
    float us;
    bool as_is;
};

float tiles_us(const TileSize& t, float count, float stages, float units) {
    const float rounds = std::floor(count / (units * t.at_once)), rest = count - rounds * units * t.at_once;
    float us = rounds * (stages * t.stage[t.at_once - 1] + t.rest[t.at_once - 1]);
    if (rest > 0) {
        const int n = std::min((int)std::ceil(rest / units), t.at_once) - 1;
        us += stages * t.stage[n] + t.rest[n];
    }
    return us;
}

// What the switches allow of that; -1: anything.
struct Pins {
    int form, splits;
    bool allows(const TileSize& t) const {
        if (form <= kDenseMemory) return true;  // those are no tiles
        const DenseForm& f = kDenseForms[form];
        return f.i == t.i && f.j == t.j && f.as_is == t.as_is;
    }
};

// The choice by `f` under the switches, without those that leave none.
template <class F>
auto pinned(const DenseCall& c, F&& f) {
    auto best = f(Pins{c.form, c.splits});
    if (best.us >= kNever && c.splits >= 0) best = f(Pins{c.form, -1});
    if (best.us >= kNever && c.form >= 0) best = f(Pins{-1, -1});
    return best;
}

// The fastest by those figures.  A sum is shared out where the last tiles would leave most of the chip idle for longer than a second
// launch, which adds up what the first left in memory, takes.  k_rows: how many of the two operands run along k.
// lay_out: us for that.
Plan plan(int dtype, int64_t I, int J, int64_t K, int k_rows, float lay_out, const Pins& pins) {
    const TileSize* const sizes = dtype == 0 ? kTilesF32 : kTiles16;
    const int count = dtype == 0 ? 4 : 7, units = compute_units(), size = dtype == 0 ? 4 : 2;
    const int64_t narrow = k_rows == 2 ? 8 : k_rows == 1 ? J : std::min<int64_t>(I, J);  // of operands that do not run along k
    const Join join = dtype == 0 ? kJoin : kJoin16;
    Plan best = {0, 0, 1, 0, kNever, false};
    for (int i = 0; i < count; ++i) {
        const TileSize& t = sizes[i];
        const int64_t tiles = ((I + t.i - 1) / t.i) * ((J + t.j - 1) / t.j), k_tiles = (K + t.depth - 1) / t.depth;
        if (tiles > kMostTiles || (t.as_is && narrow < 16 / size) || !pins.allows(t)) continue;
        const float stage = t.depth / 64.f, launch = kLaunchUs + (t.as_is ? 0.f : lay_out);
        // what tiles that read their operands as they are have on its way: 2 us for two stages of every workgroup
        const float bytes = t.as_is ? (float)(I + J) * K * size : 0.f, slots_bytes = (float)((t.i + t.j) * t.depth * size);
        const auto memory_us = [&](float workgroups) { return bytes / (std::min(workgroups, (float)units * t.at_once) * slots_bytes); };
        const float us = launch + std::max(tiles_us(t, (float)tiles, k_tiles * stage, (float)units), memory_us((float)tiles));
        if (us < best.us && pins.splits <= 1) best = {i, (int)tiles, 1, tiles, us, t.as_is};
        const int64_t slots = units * t.at_once, whole = tiles / slots * slots, shared = tiles - whole;
        const float base = launch + join.us + tiles_us(t, (float)whole, k_tiles * stage, (float)units);
        if (shared == 0) continue;
        for (int splits : {2, 3, 4, 6, 8, 12, 16, 24, 32, 48, 64}) {
            if (pins.splits == 1) break;
            if (pins.splits > 1) splits = pins.splits;
            const float moved = base + 2.f * splits * shared * t.i * t.j * 4 / join.bytes_per_us;
            if (splits > k_tiles || moved >= best.us || shared * splits > kMostTiles) break;
            const float shared_us = moved + std::max(tiles_us(t, (float)shared * splits, (float)((k_tiles + splits - 1) / splits) * stage, (float)units),
                                                     memory_us((float)tiles + (float)shared * (splits - 1)));
            if (shared_us < best.us) best = {i, (int)whole, splits, tiles, shared_us, t.as_is};
        }
    }
    return best;
}

// Both gradients' products in one launch: of one tile, and every sum of a product shared out or none.
struct PairPlan {
    int tile, x_splits, w_splits, x_first;
    int64_t x_tiles, w_tiles;
    float us;
    bool as_is;
};

PairPlan pair_plan(int dtype, int64_t N, int D, int M, float lay_out, const Pins& pins) {
    const TileSize* const sizes = dtype == 0 ? kTilesF32 : kTiles16;
    const int count = dtype == 0 ? 4 : 7;
    const float units = (float)compute_units();
    const Join join = kJoin;
    PairPlan best = {0, 1, 1, 0, 0, 0, kNever, false};
    for (int i = 0; i < count; ++i) {
        const TileSize& t = sizes[i];
        const int64_t x_tiles = ((N + t.i - 1) / t.i) * ((D + t.j - 1) / t.j), w_tiles = ((int64_t)(D + t.i - 1) / t.i) * ((M + t.j - 1) / t.j);
        if (std::max(x_tiles, w_tiles) > kMostTiles || (t.as_is && std::min(D, M) < (dtype == 0 ? 4 : 8)) || !pins.allows(t)) continue;
        const float x_stages = (float)((M + t.depth - 1) / t.depth), w_stages = (float)((N + t.depth - 1) / t.depth);
        const float unit = t.depth / 64.f, slots = units * t.at_once, tile_bytes = 8.f * t.i * t.j / join.bytes_per_us;
        for (int xs : {1, 2, 4}) {
            if (pins.splits > 0) xs = pins.splits;
            if (xs > 1 && (xs > x_stages || x_tiles > slots)) break;
            for (int ws : {1, 2, 4, 8, 16, 32}) {
                if (pins.splits > 0) ws = pins.splits;
                if (ws > 1 && (ws > w_stages || w_tiles * ws > 4 * slots)) break;
                const float nx = (float)x_tiles * xs, nw = (float)w_tiles * ws;
                const float kx = std::ceil(x_stages / xs) * unit, kw = std::ceil(w_stages / ws) * unit;
                // alone as many at once as there are; else the work by the slots, and two fifths of the longer tile for the end
                const int at_once = std::min((int)std::ceil((nx + nw) / units), t.at_once) - 1;
                const float x = kx * t.stage[at_once] + t.rest[at_once], w = kw * t.stage[at_once] + t.rest[at_once];
                float us = std::max(x, w);
                if (nx + nw > slots) us = std::max(us, (nx * x + nw * w) / slots + 0.4f * std::max(x, w));
                us += kLaunchUs + (t.as_is ? 0.f : lay_out) + (xs > 1 ? join.us + nx * tile_bytes : 0.f) + (ws > 1 ? join.us + nw * tile_bytes : 0.f);
                if (us < best.us) best = {i, xs, ws, x >= w, x_tiles, w_tiles, us, t.as_is};
            }
        }
    }
    return best;
}

size_t tile_bytes(int dtype, int tile, int64_t tiles, int splits) {
    const TileSize& t = dtype == 0 ? kTilesF32[tile] : kTiles16[tile];
    return splits > 1 ? (size_t)splits * tiles * t.i * t.j * 4 : 0;
}

size_t partial_bytes(int dtype, const Plan& p) { return tile_bytes(dtype, p.tile, p.tiles - p.whole, p.splits); }


ProductArgs product_args(const Operand& A, const Operand& B, int64_t I, int J, int64_t K, int whole, int splits, void* partial,
                         const Epilogue& e) {
    return {A, B, I, K, J, 0, 0, whole, splits, static_cast<float*>(partial), e};
}

hipError_t run(int dtype, int tile, bool a_k, bool b_k, const ProductArgs& a, hipStream_t s) {
    switch (dtype) {
        case 0: return launch_product_f32(tile, a_k, b_k, a, s);
        case 1: return launch_product_bf16(tile, a_k, b_k, a, s);
        default: return launch_product_f16(tile, a_k, b_k, a, s);
    }
}

hipError_t run(int dtype, int tile, const PairArgs& p, hipStream_t s) {
    switch (dtype) {
        case 0: return launch_pair_f32(tile, p, s);
        case 1: return launch_pair_bf16(tile, p, s);
        default: return launch_pair_f16(tile, p, s);
    }
}

unsigned lay_out_blocks(const LayOut& a) {
    int64_t units = 0;
    for (int m = 0; m < 2; ++m)
        if (a.to[m]) units += a.rows[m] * (laid_out_stride(a.width[m]) / kVec);
    return (unsigned)std::min<int64_t>((units + 255) / 256, 1 << 15);
}

hipError_t launch_lay_out(int dtype, const LayOut& a, hipStream_t s) {
    const unsigned blocks = lay_out_blocks(a);
    if (blocks == 0) return hipSuccess;
    return with_type(dtype, [&](auto t) {
        hipLaunchKernelGGL(lay_out_kernel<decltype(t)>, dim3(blocks), dim3(256), 0, s, a);
        return hipGetLastError();
    });
}

// Shares of the workspace, in the order that they are asked for.
struct Shares {
    char* at;
    void* take(size_t bytes) {
        char* const p = at;
        at += bytes;
        return p;
    }
};

// A matrix of the call as an operand: itself, or where it is laid out.  k_inner: its rows run along k.
Operand operand(const void* given, int64_t ld, const uint16_t* laid_out, int64_t rows, int64_t width, bool k_inner, bool f32) {
    const float* const origin = f32 ? static_cast<const float*>(given) : nullptr;
    Operand o = {given, ld, 0, origin, k_inner ? ld : 1, k_inner ? 1 : ld, nullptr, 0, 0, 0};
    if (laid_out) o.p = laid_out, o.ld = laid_out_stride(width), o.plane = rows * o.ld;
    return o;
}

// Whether the way straight from memory, in `plain` us, is taken in place of tiles.
bool plain_taken(const DenseCall& c, float plain, float tiles) {
    return c.dtype == 0 && (c.form > kDenseFew ? c.form == kDenseMemory && plain < kNever : plain < tiles);
}

// What the backward pass has to have laid out, and its products: of both gradients in one launch, or of one.
struct GradientPlan {
    bool plain, as_is;  // products of the operands as they are: fp32 ones without tiles, or either way
    bool x, w, z, sums, direct, pass, both;  // direct: db's sums are taken beside the products
    Plan one;
    PairPlan pair;
    SlopeArgs slope;
    size_t x_partial, partial;
};

GradientPlan gradient_plan(const DenseCall& c, const void* G, int64_t ldg, int activation, bool need_dx, bool need_dw, bool need_db) {
    GradientPlan g = {};
    g.both = need_dx && need_dw;
    float tiles = 0.f, plain = 0.f;
    const bool x_used = usable(c.dtype, c.X, c.ldx, c.D), w_used = usable(c.dtype, c.W, c.ldw, c.M), g_used = usable(c.dtype, G, ldg, c.M);
    const float values = (g_used ? 0.f : (float)c.N * c.M) + (need_dx && !w_used ? (float)c.D * c.M : 0.f) +
                         (need_dw && !x_used ? (float)c.N * c.D : 0.f);
    // the pass over G is there for an activation or a bias either way; planes are half as much again to write
    const float lay_out = lay_out_us(c.dtype, values);
    if (g.both) {
        g.pair = pinned(c, [&](const Pins& p) { return pair_plan(c.dtype, c.N, c.D, c.M, lay_out, p); });
        tiles = g.pair.us, plain = plain_pair_us(c.N, c.D, c.M), g.as_is = g.pair.as_is;
    } else if (need_dx) {
        g.one = pinned(c, [&](const Pins& p) { return plan(c.dtype, c.N, c.D, c.M, 2, lay_out, p); });
        tiles = g.one.us, plain = plain_f32_us(c.N, c.D, c.M), g.as_is = g.one.as_is;
    } else if (need_dw) {
        g.one = pinned(c, [&](const Pins& p) { return plan(c.dtype, c.D, c.M, c.N, 0, lay_out, p); });
        tiles = g.one.us, plain = plain_f32_us(c.D, c.M, c.N), g.as_is = g.one.as_is;
    }
    g.plain = plain_taken(c, plain, tiles);
    g.as_is |= g.plain;
    g.x = !g.as_is && need_dw && !x_used;
    g.w = !g.as_is && need_dx && !w_used;
    g.z = (need_dx || need_dw) && (activation != 0 || (!g.as_is && !g_used));
    // Where nothing else has to read G before the products, few rows of it are added up beside them, 32 columns per workgroup, and
    // not in a pass of their own: 256 x 768 x 768 in bf16 8.0 us for 12.0, 2048 x 768 x 768 22.7 for 23.2, 4096 x 256 x 256 23.4 for 18.3.
    g.direct = need_db && g.both && !g.z && !g.x && !g.w && c.N <= kDirectRows;
    g.sums = need_db && !g.direct;
    g.pass = g.z || g.sums;
    share_rows(c.N, c.M, g.slope);
    if (!g.plain && g.both) {
        g.x_partial = tile_bytes(c.dtype, g.pair.tile, g.pair.x_tiles, g.pair.x_splits);
        g.partial = g.x_partial + tile_bytes(c.dtype, g.pair.tile, g.pair.w_tiles, g.pair.w_splits);
    } else if (!g.plain && (need_dx || need_dw)) {
        g.partial = partial_bytes(c.dtype, g.one);
    }
    return g;
}

size_t slope_bytes(const DenseCall& c, const GradientPlan& g) {
    return g.as_is && c.dtype == 0 ? (size_t)round_up(c.N * c.M * 4, 256) : laid_out_bytes(c.dtype, c.N, c.M);
}
size_t column_bytes(const GradientPlan& g, int M) { return g.sums ? (size_t)round_up((int64_t)g.slope.chunks * M * 4, 256) : 0; }

// How a forward pass goes: few rows, plain fp32, or tiles of operands that may have to be laid out.
struct ForwardPlan {
    bool few, plain, x, w;
    Plan product;
};

ForwardPlan forward_plan(const DenseCall& c) {
    ForwardPlan f = {};
    f.few = c.form == kDenseFew ? c.N <= most_few_rows(c.dtype) : c.form < 0 && few_rows(c.dtype, c.N, c.D, c.M);
    if (f.few) return f;
    const bool x_used = usable(c.dtype, c.X, c.ldx, c.D), w_used = usable(c.dtype, c.W, c.ldw, c.M);
    const float lay_out = lay_out_us(c.dtype, (x_used ? 0.f : (float)c.N * c.D) + (w_used ? 0.f : (float)c.D * c.M));
    f.product = pinned(c, [&](const Pins& p) { return plan(c.dtype, c.N, c.M, c.D, 1, lay_out, p); });
    f.plain = plain_taken(c, plain_f32_us(c.N, c.M, c.D), f.product.us);
    f.x = !f.plain && !f.product.as_is && !x_used;
    f.w = !f.plain && !f.product.as_is && !w_used;
    return f;
}

}  // namespace

size_t dense_linear_workspace(const DenseCall& c) {
    const ForwardPlan f = forward_plan(c);
    if (f.few || f.plain) return 0;
    return (f.x ? laid_out_bytes(c.dtype, c.N, c.D) : 0) + (f.w ? laid_out_bytes(c.dtype, c.D, c.M) : 0) + partial_bytes(c.dtype, f.product);
}

hipError_t launch_dense_linear(const DenseCall& c, const float* bias, int activation, const void* R, int64_t ldr, void* Y,
                               int64_t ldy, void* Z, int64_t ldz, void* workspace, hipStream_t s) {
    const ForwardPlan f = forward_plan(c);
    const Epilogue epilogue = {bias, activation, R, Y, Z, ldr, ldy, ldz};
    if (f.few) return launch_few_rows(c.dtype, c.X, c.N, c.ldx, c.W, c.ldw, c.D, c.M, epilogue, s);
    if (f.plain)
        return launch_plain_f32({static_cast<const float*>(c.X), c.ldx, 1}, {static_cast<const float*>(c.W), 1, c.ldw}, c.N, c.M, c.D,
                                epilogue, s);
    Shares shares = {static_cast<char*>(workspace)};
    uint16_t *x = nullptr, *w = nullptr;
    if (f.x) x = static_cast<uint16_t*>(shares.take(laid_out_bytes(c.dtype, c.N, c.D)));
    if (f.w) w = static_cast<uint16_t*>(shares.take(laid_out_bytes(c.dtype, c.D, c.M)));
    if (hipError_t e = launch_lay_out(c.dtype, {{c.X, c.W}, {c.ldx, c.ldw}, {c.N, c.D}, {c.D, c.M}, {x, w}}, s)) return e;
    const bool f32 = c.dtype == 0;
    return run(c.dtype, f.product.tile, true, false,
               product_args(operand(c.X, c.ldx, x, c.N, c.D, true, f32), operand(c.W, c.ldw, w, c.D, c.M, false, f32), c.N, c.M, c.D,
                            f.product.whole, f.product.splits, shares.take(0), epilogue),
               s);
}

size_t dense_linear_gradient_workspace(const DenseCall& c, const void* G, int64_t ldg, const void*, int64_t, int activation,
                                       bool need_dx, bool need_dw, bool need_db) {
    const GradientPlan g = gradient_plan(c, G, ldg, activation, need_dx, need_dw, need_db);
    return (g.x ? laid_out_bytes(c.dtype, c.N, c.D) : 0) + (g.w ? laid_out_bytes(c.dtype, c.D, c.M) : 0) +
           (g.z ? slope_bytes(c, g) : 0) + column_bytes(g, c.M) + g.partial;
}

hipError_t launch_dense_linear_gradient(const DenseCall& c, const void* G, int64_t ldg, const void* Z, int64_t ldz, int activation,
                                        void* dX, int64_t lddx, void* dW, int64_t lddw, float* db, void* workspace,
                                        hipStream_t s) {
    if (c.N == 0) return launch_clear(c.dtype, dW, lddw, c.D, c.M, db, s);
    GradientPlan g = gradient_plan(c, G, ldg, activation, dX, dW, db);
    Shares shares = {static_cast<char*>(workspace)};
    uint16_t *x = nullptr, *w = nullptr, *z = nullptr;
    if (g.x) x = static_cast<uint16_t*>(shares.take(laid_out_bytes(c.dtype, c.N, c.D)));
    if (g.w) w = static_cast<uint16_t*>(shares.take(laid_out_bytes(c.dtype, c.D, c.M)));
    if (g.z) z = static_cast<uint16_t*>(shares.take(slope_bytes(c, g)));
    float* const columns = static_cast<float*>(shares.take(column_bytes(g, c.M)));
    float *const x_partial = static_cast<float*>(shares.take(g.x_partial)), *const w_partial = static_cast<float*>(shares.take(0));
    const LayOut others = {{c.X, c.W}, {c.ldx, c.ldw}, {c.N, c.D}, {c.D, c.M}, {x, w}};
    if (g.pass) {
        SlopeArgs& a = g.slope;
        a.G = G, a.Z = Z, a.ldg = ldg, a.ldz = ldz, a.N = c.N, a.M = c.M, a.activation = activation;
        a.to = z, a.plain = g.as_is && c.dtype == 0, a.partial = g.sums ? columns : nullptr;
        const hipError_t e = with_type(c.dtype, [&](auto t) {
            hipLaunchKernelGGL(slope_kernel<decltype(t)>, dim3((unsigned)(a.chunks * a.col_tiles) + lay_out_blocks(others)), dim3(256), 0, s,
                               a, others);
            return hipGetLastError();
        });
        if (e != hipSuccess) return e;
    } else if (hipError_t e = launch_lay_out(c.dtype, others, s)) {
        return e;
    }
    const PartialSums sums = g.direct ? PartialSums{nullptr, (int)c.N, c.M, db, G, ldg} : PartialSums{columns, g.slope.chunks, c.M, db, nullptr, 0};
    if (!g.both && db)
        if (hipError_t e = launch_partial_sums(columns, g.slope.chunks, c.M, c.M, db, nullptr, s)) return e;
    if (!dX && !dW) return hipSuccess;
    const Epilogue to_x = {nullptr, 0, nullptr, dX, nullptr, 0, lddx, 0}, to_w = {nullptr, 0, nullptr, dW, nullptr, 0, lddw, 0};
    if (g.plain) {
        const float *const dz = static_cast<const float*>(g.z ? static_cast<const void*>(z) : G), *const X = static_cast<const float*>(c.X),
                    *const W = static_cast<const float*>(c.W);
        const int64_t ld = g.z ? c.M : ldg;
        if (g.both) return launch_plain_pair_f32(dz, ld, W, c.ldw, X, c.ldx, c.N, c.D, c.M, to_x, to_w, sums, s);
        return dX ? launch_plain_f32({dz, ld, 1}, {W, c.ldw, 1}, c.N, c.D, c.M, to_x, s)
                  : launch_plain_f32({X, 1, c.ldx}, {dz, 1, ld}, c.D, c.M, c.N, to_w, s);
    }
    const bool f32 = c.dtype == 0;
    const auto gradient = [&](bool k_inner) {
        if (g.as_is && z && f32) return operand(z, c.M, nullptr, c.N, c.M, k_inner, f32);
        Operand o = operand(G, ldg, z, c.N, c.M, k_inner, f32);
        if (f32 && activation) {
            o.slope_of = static_cast<const float*>(Z), o.activation = activation;
            o.slope_outer = k_inner ? ldz : 1, o.slope_k = k_inner ? 1 : ldz;
        }
        return o;
    };
    const auto product = [&](bool of_x, int whole, int splits, float* partial) {
        return of_x ? product_args(gradient(true), operand(c.W, c.ldw, w, c.D, c.M, true, f32), c.N, c.D, c.M, whole, splits, partial, to_x)
                    : product_args(operand(c.X, c.ldx, x, c.N, c.D, false, f32), gradient(false), c.D, c.M, c.N, whole, splits, partial, to_w);
    };
    if (!g.both) return run(c.dtype, g.one.tile, dX != nullptr, dX != nullptr, product(dX, g.one.whole, g.one.splits, w_partial), s);
    const PairPlan& p = g.pair;
    return run(c.dtype, p.tile,
               {product(true, p.x_splits > 1 ? 0 : (int)p.x_tiles, p.x_splits, x_partial),
                product(false, p.w_splits > 1 ? 0 : (int)p.w_tiles, p.w_splits, w_partial), 0, 0, p.x_first, sums},
               s);
}

}  // namespace lutnn
