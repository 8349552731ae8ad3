// The matrix products of dense linear layers on the matrix cores, C[i][j] = sum_k A(i, k) B(k, j), with the layer's epilogue.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "activation.h"
#include "lutnn_kernels.h"
#include "matrix_types.h"
#include "mfma_tile.h"
#include "split_bf16.h"

namespace lutnn {

// What becomes of a sum: bias, activation and residual; Z receives it before the activation.
struct Epilogue {
    const float* bias;
    int activation;
    const void* R;
    void* Y;
    void* Z;
    int64_t ldr, ldy, ldz;
};

// An operand as the kernel reads it: 16-bit values, rows of `ld` of them in whole aligned 16-byte units, zeros behind a row's end as
// far as its unit goes; PARTS planes.
struct Operand {
    const void* p;
    int64_t ld, plane;  // values
    // fp32 operands: where the planes come from, the value at outer index o and k being origin[o * step_outer + k * step_k], times
    // the activation's slope at slope_of[o * slope_outer + k * slope_k]
    const float* origin;
    int64_t step_outer, step_k;
    const float* slope_of;
    int64_t slope_outer, slope_k;
    int activation;
};

struct ProductArgs {
    Operand A, B;
    int64_t I, K;
    int J, i_tiles, j_tiles, splits;
    float* partial;  // [splits][I][J] where splits > 1
    Epilogue e;
};

namespace product {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef short s16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));

constexpr uint32_t kBeyond = 0xc0000000u;  // an offset past any tile's rows: the load gives zeros

__device__ __forceinline__ f32x4 mfma(s16x8 a, s16x8 b, f32x4 c, bf16) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}
__device__ __forceinline__ f32x4 mfma(s16x8 a, s16x8 b, f32x4 c, f16) {
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
}

// Orders the workgroup's LDS operations only: loads to LDS stay in flight.
__device__ __forceinline__ void lds_barrier() {
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup", "local");
    __builtin_amdgcn_s_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup", "local");
}

// 64 lanes x 16 bytes from the buffer `rsrc` straight into LDS at lds_dst + 16 * lane; zeros for offsets past its end.
__device__ __forceinline__ void buffer_to_lds(uint32_t lds_dst, i32x4 rsrc, uint32_t voff) {
    asm volatile(
        "s_mov_b32 m0, %0\n\t"
        "s_nop 0\n\t"
        "buffer_load_dwordx4 %1, %2, 0 offen lds"
        :
        : "s"(lds_dst), "v"(voff), "s"(rsrc)
        : "memory", "m0");
}

// One operand's tile: `OUT` rows (of A) or columns (of B) by DEPTH k.  K_INNER: k is contiguous in memory, and a tile is OUT rows
// of DEPTH values in LDS; otherwise DEPTH rows of OUT values, which the transposing LDS reads turn.
template <int OUT, int DEPTH, bool K_INNER, int PARTS, int THREADS>
struct Tile {
    static constexpr int kRow = K_INNER ? DEPTH : OUT;             // values of a row in LDS
    static constexpr int kUnits = kRow / 8;                        // 16-byte units of it
    static constexpr int kPart = OUT * DEPTH * 2;                  // bytes
    static constexpr int kBytes = kPart * PARTS;
    static constexpr int kLoads = kPart / (THREADS * 16);          // per thread and part
    static_assert(kPart % (THREADS * 16) == 0, "whole loads");

    // Where unit u of a row lies in it.  k inner: rows of 128 or 64 bytes, read 16 of them at a time at one unit; the same unit of
    // eight (four) neighbouring rows lies in different banks.  Otherwise rows k .. k + 3 of each of four groups eight apart are read
    // at once, 32 bytes of each: pairs of units are moved.
    static __device__ __forceinline__ int place(int row, int u) {
        if constexpr (K_INNER) return kUnits == 8 ? u ^ (row & 7) : u ^ ((row >> 1) & 3);
        if constexpr (kUnits >= 16) return u ^ (((row & 3) | ((row >> 1) & 4)) << 1);
        return u ^ ((row & 3) << 1);
    }

    const char* base;   // of the tile's first row, k = 0
    int64_t plane;      // bytes
    int64_t k_step;     // bytes from one k tile to the next
    uint32_t stride, width;  // bytes: of a row, and where k is not inner from the tile's first value to the end of its row
    uint32_t off[kLoads];
    int64_t K;          // where it is inner, in whole units: rows end in zeros as far as that
    int64_t rows;       // of the operand from the tile's first one on, where k is inner

    __device__ __forceinline__ Tile(const Operand& o, int64_t first, int64_t count, int64_t K_)
        : K(K_INNER ? (K_ + 7) / 8 * 8 : K_) {
        stride = (uint32_t)(o.ld * 2);
        plane = o.plane * 2;
        if constexpr (K_INNER) {
            base = static_cast<const char*>(o.p) + first * o.ld * 2;
            rows = min((int64_t)OUT, count - first);
            k_step = DEPTH * 2;
        } else {
            base = static_cast<const char*>(o.p) + first * 2;
            k_step = (int64_t)DEPTH * stride;
            width = (uint32_t)(min((int64_t)OUT, (count - first + 7) / 8 * 8) * 2);
        }
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            const int slot = i * THREADS + threadIdx.x, row = slot / kUnits;
            off[i] = (uint32_t)row * stride + (uint32_t)place(row, slot % kUnits) * 16;
        }
    }

    // Loads k tile t into LDS at `to`.
    __device__ __forceinline__ void load(uint32_t to, int64_t t) const {
        const int64_t left = K - t * DEPTH;  // > 0
        const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
        uint32_t end;
        if constexpr (K_INNER)
            end = (uint32_t)(rows - 1) * stride + (uint32_t)min(left, (int64_t)DEPTH) * 2;
        else
            end = (uint32_t)(min(left, (int64_t)DEPTH) - 1) * stride + width;
#pragma unroll
        for (int p = 0; p < PARTS; ++p) {
            const uint64_t at = reinterpret_cast<uint64_t>(base + p * plane + t * k_step);
            const i32x4 rsrc = {(int)(uint32_t)at, (int)(uint32_t)(at >> 32), (int)end, 0x00020000};
#pragma unroll
            for (int i = 0; i < kLoads; ++i) {
                uint32_t o = off[i];
                if constexpr (K_INNER) {
                    if (left < DEPTH) {  // past the last k of a row: not the next row's values, but zeros
                        const int slot = i * THREADS + threadIdx.x, row = slot / kUnits;
                        if (place(row, slot % kUnits) * 8 >= left) o = kBeyond;
                    }
                }
                buffer_to_lds(to + p * kPart + i * THREADS * 16 + wave * 1024, rsrc, o);
            }
        }
    }

    // The matrix instruction's operand for outer index first + lane % 16 and k = 32 s + 8 (lane / 16) .. + 7.
    static __device__ __forceinline__ s16x8 fragment(const char* part, int first, int s) {
        const int lane = threadIdx.x & 63, i = lane & 15, q = lane >> 4;
        if constexpr (K_INNER) {
            const int row = first + i;
            return *reinterpret_cast<const s16x8*>(part + row * kRow * 2 + place(row, 4 * s + q) * 16);
        } else {
            typedef __attribute__((address_space(3))) s16x4* lds4;
            s16x4 half[2];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int row = 32 * s + 8 * q + 4 * h + (i >> 2);
                const char* const at = part + row * kRow * 2 + place(row, first / 8 + ((i & 3) >> 1)) * 16 + (i & 1) * 8;
                half[h] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4)(at));
            }
            return __builtin_shufflevector(half[0], half[1], 0, 1, 2, 3, 4, 5, 6, 7);
        }
    }
};

// A sum that the parts could not form, as one fp32 chain.
__device__ __forceinline__ float chain(const ProductArgs& a, int64_t i, int64_t j) {
    const auto value = [](const Operand& o, int64_t outer, int64_t k) {
        const float v = o.origin[outer * o.step_outer + k * o.step_k];
        return o.slope_of ? v * slope(o.slope_of[outer * o.slope_outer + k * o.slope_k], o.activation) : v;
    };
    float sum = 0.f;
#pragma unroll 1
    for (int64_t k = 0; k < a.K && sum == sum; ++k) sum = __fmaf_rn(value(a.A, i, k), value(a.B, j, k), sum);
    return sum;
}

// `n` sums of one row, or fewer at the right edge, through the epilogue.
template <class T, int n>
__device__ __forceinline__ void finish(const Epilogue& e, int64_t i, int j, int J, float (&z)[n]) {
    if (j + n <= J) {
        if (e.bias) {
            float b[n];
            load_values(e.bias + j, b);
#pragma unroll
            for (int r = 0; r < n; ++r) z[r] += b[r];
        }
        if (e.Z) store_values(static_cast<T*>(e.Z) + i * e.ldz + j, z);
        float x[n] = {};
        if (e.R) load_values(static_cast<const T*>(e.R) + i * e.ldr + j, x);
        activate_all(z, e.activation);
#pragma unroll
        for (int r = 0; r < n; ++r) z[r] += x[r];
        store_values(static_cast<T*>(e.Y) + i * e.ldy + j, z);
        return;
    }
    T *const Z = static_cast<T*>(e.Z), *const Y = static_cast<T*>(e.Y);
#pragma unroll
    for (int r = 0; r < n; ++r) {
        if (j + r >= J) break;
        if (e.bias) z[r] += e.bias[j + r];
        if (Z) Z[i * e.ldz + j + r] = (T)z[r];
    }
    activate_all(z, e.activation);
#pragma unroll
    for (int r = 0; r < n; ++r) {
        if (j + r >= J) break;
        if (e.R) z[r] += (float)static_cast<const T*>(e.R)[i * e.ldr + j + r];
        Y[i * e.ldy + j + r] = (T)z[r];
    }
}

// One tile per workgroup.  T: the matrices' type; fp32 ones are PARTS = 3 planes of bf16 (split_bf16.h).  WI x WJ wavefronts.
template <class T, int TI, int TJ, int WI, int WJ, bool A_K, bool B_K>
__global__ __launch_bounds__(64 * WI * WJ) void product_kernel(ProductArgs a) {
    constexpr bool F32 = sizeof(T) == 4;
    constexpr int PARTS = F32 ? 3 : 1, DEPTH = F32 ? 32 : 64, THREADS = 64 * WI * WJ;
    constexpr int FI = TI / WI / 16, FJ = TJ / WJ / 16;
    typedef typename std::conditional<F32, bf16, T>::type E;
    typedef Tile<TI, DEPTH, A_K, PARTS, THREADS> TileA;
    typedef Tile<TJ, DEPTH, B_K, PARTS, THREADS> TileB;
    constexpr int BUF = TileA::kBytes + TileB::kBytes;
    // the sums on their way out: a wavefront's, ROUND rows at a time
    constexpr int ROUND = TI / WI < 64 ? TI / WI : 64, COLS = TJ / WJ, PITCH = COLS + 4, OUT = WI * WJ * ROUND * PITCH * 4;
    __shared__ __align__(1024) char lds[2 * BUF > OUT ? 2 * BUF : OUT];

    // neighbouring tiles on one XCD: groups of four rows of tiles, column by column
    const int64_t tiles = (int64_t)a.i_tiles * a.j_tiles;
    const int64_t tile = xcd_tile(tiles * a.splits);
    if (tile < 0) return;
    const int split = (int)(tile / tiles), in_split = (int)(tile % tiles);
    const int group = in_split / (4 * a.j_tiles), rest = in_split % (4 * a.j_tiles);
    const int group_rows = min(4, a.i_tiles - 4 * group);
    const int64_t i0 = (int64_t)(4 * group + rest % group_rows) * TI;
    const int j0 = rest / group_rows * TJ;

    const TileA ta(a.A, i0, a.I, a.K);
    const TileB tb(a.B, j0, a.J, a.K);
    const int64_t k_tiles = (a.K + DEPTH - 1) / DEPTH;
    const int64_t t0 = k_tiles * split / a.splits, t1 = k_tiles * (split + 1) / a.splits;

    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wi = wave / WJ * (TI / WI), wj = wave % WJ * (TJ / WJ);
    f32x4 sum[FI][FJ];
#pragma unroll
    for (int i = 0; i < FI; ++i)
#pragma unroll
        for (int j = 0; j < FJ; ++j) sum[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};

    const uint32_t base = lds_offset(lds);
    if (t0 < t1) {
        ta.load(base, t0);
        tb.load(base + TileA::kBytes, t0);
    }
    for (int64_t t = t0; t < t1; ++t) {
        const int cur = (int)(t - t0) & 1;
        wait_loads<0>();
        lds_barrier();  // everybody's loads are there, and everybody has read the other buffer
        if (t + 1 < t1) {
            ta.load(base + (cur ^ 1) * BUF, t + 1);
            tb.load(base + (cur ^ 1) * BUF + TileA::kBytes, t + 1);
        }
        const char* const pa = lds + cur * BUF;
        const char* const pb = pa + TileA::kBytes;
#pragma unroll
        for (int s = 0; s < DEPTH / 32; ++s) {
            if constexpr (!F32) {
                s16x8 fa[FI], fb[FJ];
#pragma unroll
                for (int j = 0; j < FJ; ++j) fb[j] = TileB::fragment(pb, wj + 16 * j, s);
#pragma unroll
                for (int i = 0; i < FI; ++i) fa[i] = TileA::fragment(pa, wi + 16 * i, s);
#pragma unroll
                for (int i = 0; i < FI; ++i)
#pragma unroll
                    for (int j = 0; j < FJ; ++j) sum[i][j] = mfma(fb[j], fa[i], sum[i][j], E());
            } else {
                constexpr int kPairs[6][2] = {{2, 0}, {0, 2}, {1, 1}, {1, 0}, {0, 1}, {0, 0}};  // small products first
                s16x8 fb[FJ][3];
#pragma unroll
                for (int j = 0; j < FJ; ++j)
#pragma unroll
                    for (int p = 0; p < 3; ++p) fb[j][p] = TileB::fragment(pb + p * TileB::kPart, wj + 16 * j, s);
#pragma unroll
                for (int i = 0; i < FI; ++i) {
                    s16x8 fa[3];
#pragma unroll
                    for (int p = 0; p < 3; ++p) fa[p] = TileA::fragment(pa + p * TileA::kPart, wi + 16 * i, s);
                    f32x4 slice[FJ];
#pragma unroll
                    for (int j = 0; j < FJ; ++j) slice[j] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                    for (int n = 0; n < 6; ++n)
#pragma unroll
                        for (int j = 0; j < FJ; ++j) slice[j] = mfma(fb[j][kPairs[n][1]], fa[kPairs[n][0]], slice[j], E());
#pragma unroll
                    for (int j = 0; j < FJ; ++j) sum[i][j] += slice[j];
                }
            }
        }
    }

    // Out through LDS, so that a row's values leave in whole lines: every wavefront its own, nothing to wait for but that all
    // have read their operands.
    lds_barrier();
    constexpr int VEC = F32 ? 4 : 8, LANES = COLS / VEC;  // values per lane, lanes per row
    const int lane = threadIdx.x & 63;
    float* const out = reinterpret_cast<float*>(lds) + wave * ROUND * PITCH;
#pragma unroll
    for (int round = 0; round < TI / WI / ROUND; ++round) {
#pragma unroll
        for (int i = 0; i < ROUND / 16; ++i)
#pragma unroll
            for (int j = 0; j < FJ; ++j) {
                f32x4 z = sum[round * ROUND / 16 + i][j];
                if constexpr (F32) z *= kUnscale;
                *reinterpret_cast<f32x4*>(out + (16 * i + (lane & 15)) * PITCH + 16 * j + 4 * (lane >> 4)) = z;
            }
        const int col = j0 + wj + lane % LANES * VEC;
#pragma unroll 1
        for (int r = lane / LANES; r < ROUND; r += 64 / LANES) {
            const int64_t row = i0 + wi + round * ROUND + r;
            if (row >= a.I || col >= a.J) continue;
            float z[VEC];
            load_values(out + r * PITCH + lane % LANES * VEC, z);
            if (a.splits > 1) {
                float* const to = a.partial + ((int64_t)split * a.I + row) * a.J + col;
                if (col + VEC <= a.J)
                    store_values(to, z);
                else
                    for (int c = 0; c < VEC && col + c < a.J; ++c) to[c] = z[c];
                continue;
            }
            if constexpr (F32)
#pragma unroll
                for (int c = 0; c < VEC; ++c)
                    if (!is_finite(z[c])) z[c] = chain(a, row, min(col + c, a.J - 1));
            finish<T>(a.e, row, col, a.J, z);
        }
    }
}

// The splits' sums through the epilogue, four columns per thread.
template <class T>
__global__ __launch_bounds__(256) void join_kernel(ProductArgs a) {
    const int quads = (a.J + 3) / 4;
    for (int64_t v = blockIdx.x * 256LL + threadIdx.x; v < a.I * quads; v += gridDim.x * 256LL) {
        const int64_t i = v / quads;
        const int j = (int)(v - i * quads) * 4;
        float z[4] = {};
        for (int s = 0; s < a.splits; ++s) {
            const float* const from = a.partial + ((int64_t)s * a.I + i) * a.J + j;
            if (j + 3 < a.J) {
                float x[4];
                load_values(from, x);
#pragma unroll
                for (int r = 0; r < 4; ++r) z[r] += x[r];
            } else {
#pragma unroll
                for (int r = 0; r < 4; ++r) z[r] += j + r < a.J ? from[r] : 0.f;
            }
        }
        if constexpr (sizeof(T) == 4)
#pragma unroll
            for (int r = 0; r < 4; ++r)
                if (!is_finite(z[r])) z[r] = chain(a, i, min(j + r, a.J - 1));
        finish<T>(a.e, i, j, a.J, z);
    }
}

template <class T, int TI, int TJ, int WI, int WJ, bool A_K, bool B_K>
hipError_t launch(ProductArgs a, hipStream_t s) {
    const int64_t i_tiles = (a.I + TI - 1) / TI;
    a.j_tiles = (a.J + TJ - 1) / TJ;
    const int64_t blocks = (i_tiles * a.j_tiles * a.splits + 7) / 8 * 8;
    if (blocks > 0x7fffffffLL) return hipErrorInvalidValue;
    a.i_tiles = (int)i_tiles;
    hipLaunchKernelGGL((product_kernel<T, TI, TJ, WI, WJ, A_K, B_K>), dim3((unsigned)blocks), dim3(64 * WI * WJ), 0, s, a);
    if (hipError_t e = hipGetLastError(); e != hipSuccess || a.splits == 1) return e;
    const int64_t quads = (a.J + 3) / 4 * a.I;
    hipLaunchKernelGGL(join_kernel<T>, dim3((unsigned)std::min<int64_t>((quads + 255) / 256, 1 << 16)), dim3(256), 0, s, a);
    return hipGetLastError();
}

template <class T>
hipError_t launch_tile(int tile, bool a_k, bool b_k, const ProductArgs& a, hipStream_t s) {
    const auto with = [&](auto ak, auto bk) {
        constexpr bool AK = decltype(ak)::value, BK = decltype(bk)::value;
        if constexpr (sizeof(T) == 4) {
            switch (tile) {
                case 0: return launch<T, 128, 128, 2, 2, AK, BK>(a, s);
                default: return launch<T, 64, 64, 2, 2, AK, BK>(a, s);
            }
        } else {
            switch (tile) {
                case 0: return launch<T, 256, 256, 2, 4, AK, BK>(a, s);
                case 1: return launch<T, 128, 128, 2, 2, AK, BK>(a, s);
                default: return launch<T, 64, 64, 2, 2, AK, BK>(a, s);
            }
        }
    };
    if (!a_k) return with(std::false_type(), std::false_type());
    return b_k ? with(std::true_type(), std::true_type()) : with(std::true_type(), std::false_type());
}

}  // namespace product

// dense_product_f32.hip, _bf16.hip, _f16.hip; tile: a size of dense_linear.hip's list.  A's k is inner but for dW = X^T dZ, B's for
// dX = dZ W^T.
hipError_t launch_product_f32(int tile, bool a_k, bool b_k, const ProductArgs& a, hipStream_t s);
hipError_t launch_product_bf16(int tile, bool a_k, bool b_k, const ProductArgs& a, hipStream_t s);
hipError_t launch_product_f16(int tile, bool a_k, bool b_k, const ProductArgs& a, hipStream_t s);

}  // namespace lutnn
