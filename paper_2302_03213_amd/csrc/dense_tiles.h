// What the kernels of the dense layers' matrix products share: their arguments, which workgroup computes which tile, and the order of
// LDS reads and matrix instructions.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "dense_epilogue.h"
#include "dense_rows.h"
#include "matrix_types.h"
#include "mfma_tile.h"
#include "split_bf16.h"

namespace lutnn {

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
    int J, i_tiles, j_tiles;
    int whole, splits;  // so many tiles are one workgroup's each; `splits` share the sum of each of the others
    float* partial;     // theirs: [splits][tiles - whole][rows of a tile][columns of it]
    Epilogue e;
};

// Both gradients' products in one launch (product::pair_kernel).
struct PairArgs {
    ProductArgs x, w;
    int x_blocks, w_blocks, x_first;  // the blocks are counted at the launch
    PartialSums sums;
};

namespace product {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef short s16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));

// 32 k of 16 rows and columns, eight per lane.
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

// Workgroup b's tile of `tiles`, -1 for none: consecutive workgroups run on different XCDs, and each of the eight takes a
// contiguous range.
__device__ __forceinline__ int of_xcd(int b, int tiles) {
    const int t = (b & 7) * ((tiles + 7) / 8) + (b >> 3);
    return t < tiles ? t : -1;
}

// Where a tile lies: groups of four rows of tiles, column by column, so that neighbours read the same rows and columns.
struct TilePlace {
    int i, j;
};
__device__ __forceinline__ TilePlace place_of(int tile, int i_tiles, int j_tiles) {
    const int group = tile / (4 * j_tiles), rest = tile % (4 * j_tiles), rows = min(4, i_tiles - 4 * group);
    return {4 * group + rest % rows, rest / rows};
}

// What workgroup `block` computes: a tile (-1 for none) and its share of the sum; slot: where that lies among the partial sums.
struct Share {
    int tile, split, splits;
    int64_t slot;
};
__device__ __forceinline__ Share share_of(const ProductArgs& a, int block) {
    const int whole_blocks = (a.whole + 7) / 8 * 8, shared = a.i_tiles * a.j_tiles - a.whole;
    if (block < whole_blocks) return {of_xcd(block, a.whole), 0, 1, 0};
    const int t = of_xcd(block - whole_blocks, shared * a.splits);
    return {t < 0 ? -1 : a.whole + t % shared, t / shared, a.splits, t};
}

// Asks for the LDS reads of a block between the first `products` of its matrix instructions, in `groups` groups of both.
template <int reads, int products, int groups, int g = 0>
__device__ __forceinline__ void interleave() {
    if constexpr (g < groups) {
        constexpr int r = reads * (g + 1) / groups - reads * g / groups, m = products * (g + 1) / groups - products * g / groups;
        if constexpr (r > 0) __builtin_amdgcn_sched_group_barrier(0x100, r, 0);
        if constexpr (m > 0) __builtin_amdgcn_sched_group_barrier(0x008, m, 0);
        interleave<reads, products, groups, g + 1>();
    }
}

}  // namespace product
}  // namespace lutnn
