// Products of fp32 operands as they are, on the fp32 matrix instructions: for layers of some hundred rows, where laying the planes of
// dense_product.h out takes longer than their faster products save.
//
// What bounds it is the instructions, 614 GFLOP/s a compute unit: a 64 x 64 tile by 32 k takes 0.48 us of 0.43.  256 x 768 x 768
// 7.7 us (planes 20; straight from memory 10.7), 1024 x 768 x 768 15 (planes 29), 256 x 2048 x 2048 23 (planes 32); from
// 2048 x 1024 x 1024 (39 and 40) on the planes are faster.  Values go through registers to LDS, two stages ahead of that, so that
// rows of any alignment are read 16 bytes at a time: four stages took 8 % longer, a third of it the first loads, but for a few
// rows by a W past the caches (64 x 4096 x 4096 26 us for 34; the sum is shared out there, 25).  A stage's operands are read from LDS
// while the last one's products run (18 % faster than behind its barrier, for the 64 x 64 tile).  Wider tiles leave too few
// workgroups where this is used; 64 x 32 is no faster than 32 x 32.
#pragma once
#include <type_traits>

#include "dense_tiles.h"
#include "matrix_types.h"

namespace lutnn {
namespace product {

// 16-byte units of one operand's tile, OUT outer indices by DEPTH k, on their way from memory to LDS through registers.  An
// operand whose rows do not run along k has four outer indices at least.
template <int OUT, int DEPTH, bool K_INNER, int THREADS>
struct Panel {
    static constexpr int kLoads = OUT * DEPTH / 4 / THREADS, kInRow = (K_INNER ? DEPTH : OUT) / 4;  // units
    static constexpr int kFront = K_INNER ? 0 : 4;  // of a row in LDS
    static constexpr int kPitch = (K_INNER ? DEPTH : OUT) + 4, kFloats = kPitch * (K_INNER ? OUT : DEPTH);
    static_assert(kLoads * THREADS * 4 == OUT * DEPTH, "whole loads");

    const float* at[kLoads];
    int to[kLoads];
    int64_t step;

    __device__ __forceinline__ Panel(const Operand& o, int64_t first, int64_t count, int64_t k0) {
        const float* const p = static_cast<const float*>(o.p);
        step = K_INNER ? DEPTH : DEPTH * o.ld;
#pragma unroll
        for (int l = 0; l < kLoads; ++l) {
            const int u = l * THREADS + threadIdx.x, row = u / kInRow;
            int col = u % kInRow * 4;
            if constexpr (K_INNER) {
                at[l] = p + min(first + row, count - 1) * o.ld + k0 + col;
            } else {  // units past the last column are moved back to end with it, repeating others' values, up to three
                      // columns in front of the tile
                col = (int)min((int64_t)col, count - 4 - first);
                at[l] = p + (k0 + row) * o.ld + first + col;
            }
            to[l] = row * kPitch + kFront + col;
        }
    }

    // left: the values of k from this tile on; what lies behind them becomes zero.
    template <bool WHOLE>
    __device__ __forceinline__ void load(f32x4 (&v)[kLoads], int left) {
#pragma unroll
        for (int l = 0; l < kLoads; ++l) {
            const int u = l * THREADS + threadIdx.x;
            if constexpr (WHOLE) {
                v[l] = *reinterpret_cast<const Packed<float, 4>::type*>(at[l]);
            } else if constexpr (K_INNER) {
                const int k = u % kInRow * 4;
#pragma unroll
                for (int r = 0; r < 4; ++r) v[l][r] = k + r < left ? at[l][r] : 0.f;
            } else {
                const int k = u / kInRow;
                v[l] = f32x4{0.f, 0.f, 0.f, 0.f};
                if (k < left) v[l] = *reinterpret_cast<const Packed<float, 4>::type*>(at[l]);
            }
            at[l] += step;
        }
    }

    __device__ __forceinline__ void store(const f32x4 (&v)[kLoads], float* panel) const {
        typedef typename std::conditional<K_INNER, f32x4, Packed<float, 4>::type>::type Unit;
#pragma unroll
        for (int l = 0; l < kLoads; ++l) *reinterpret_cast<Unit*>(panel + to[l]) = v[l];
    }

    // Four k of 16 outer indices from `first` on: those from k + 4 q on in lane group q.
    static __device__ __forceinline__ f32x4 fragment(const float* panel, int first, int k) {
        const int lane = threadIdx.x & 63, outer = first + (lane & 15), from = k + lane / 16 * 4;
        if constexpr (K_INNER) return *reinterpret_cast<const f32x4*>(panel + outer * kPitch + from);
        f32x4 v;
#pragma unroll
        for (int r = 0; r < 4; ++r) v[r] = panel[(from + r) * kPitch + kFront + outer];
        return v;
    }
};

// As Config of dense_product.h.  WAVES: of a SIMD unit, at least; what the registers have to leave room for.
template <int TI_, int TJ_, int WI_, int WJ_, int DEPTH_, int WAVES_>
struct ConfigF32 {
    typedef float T;
    static constexpr bool AS_IS = true;
    static constexpr int TI = TI_, TJ = TJ_, WI = WI_, WJ = WJ_, DEPTH = DEPTH_, THREADS = 64 * WI * WJ, WAVES = WAVES_;
    static constexpr int floats(int out) { return out * DEPTH + 4 * (out > DEPTH ? out : DEPTH); }
    static constexpr int LDS = 2 * 4 * (floats(TI) + floats(TJ));
};

// Workgroup `block`'s tile.  Stage t + 1's operands are read from LDS, stage t + 2's written there and stage t + 4's asked for while
// stage t's are multiplied.
template <class C, bool A_K, bool B_K>
__device__ __forceinline__ void tile_f32(const ProductArgs& a, int block, char* const lds) {
    constexpr int TI = C::TI, TJ = C::TJ, DEPTH = C::DEPTH, FI = TI / C::WI / 16, FJ = TJ / C::WJ / 16, AHEAD = 2, STEPS = DEPTH / 16;
    typedef Panel<TI, DEPTH, A_K, C::THREADS> PanelA;
    typedef Panel<TJ, DEPTH, B_K, C::THREADS> PanelB;
    constexpr int BUF = PanelA::kFloats + PanelB::kFloats;
    static_assert(2 * BUF * 4 <= C::LDS, "two buffers");
    const Share share = share_of(a, block);
    if (share.tile < 0) return;
    const TilePlace place = place_of(share.tile, a.i_tiles, a.j_tiles);
    const int64_t i0 = (int64_t)place.i * TI;
    const int j0 = place.j * TJ;
    const int k_tiles = (int)((a.K + DEPTH - 1) / DEPTH);
    const int t0 = (int)((int64_t)k_tiles * share.split / share.splits);
    const int stages = (int)((int64_t)k_tiles * (share.split + 1) / share.splits) - t0;
    const int k_left = (int)min(a.K - (int64_t)t0 * DEPTH, (int64_t)stages * DEPTH), whole = k_left / DEPTH;
    PanelA pa(a.A, i0, a.I, (int64_t)t0 * DEPTH);
    PanelB pb(a.B, j0, a.J, (int64_t)t0 * DEPTH);
    const int wave = threadIdx.x >> 6, wi = wave / C::WJ * (TI / C::WI), wj = wave % C::WJ * (TJ / C::WJ);
    float* const buffers = reinterpret_cast<float*>(lds);

    struct Stage {
        f32x4 a[PanelA::kLoads], b[PanelB::kLoads];
    };
    Stage ring[AHEAD];
    f32x4 sum[FI][FJ] = {};
    const auto load = [&](Stage& s, int t) {
        if (t < whole) {
            pa.template load<true>(s.a, 0);
            pb.template load<true>(s.b, 0);
        } else if (t < stages) {
            pa.template load<false>(s.a, k_left - t * DEPTH);
            pb.template load<false>(s.b, k_left - t * DEPTH);
        }
    };
    const auto store = [&](const Stage& s, int t) {
        float* const to = buffers + (t & 1) * BUF;
        pa.store(s.a, to);
        pb.store(s.b, to + PanelA::kFloats);
    };
    struct Fragments {
        f32x4 a[STEPS][FI], b[STEPS][FJ];
    };
    const auto read = [&](Fragments& f, int t) {
        const float *const at = buffers + (t & 1) * BUF, *const bt = at + PanelA::kFloats;
#pragma unroll
        for (int k = 0; k < STEPS; ++k) {
#pragma unroll
            for (int i = 0; i < FI; ++i) f.a[k][i] = PanelA::fragment(at, wi + 16 * i, 16 * k);
#pragma unroll
            for (int j = 0; j < FJ; ++j) f.b[k][j] = PanelB::fragment(bt, wj + 16 * j, 16 * k);
        }
    };
    const auto multiply = [&](const Fragments& f) {
#pragma unroll
        for (int k = 0; k < STEPS; ++k)
#pragma unroll
            for (int r = 0; r < 4; ++r)
#pragma unroll
                for (int i = 0; i < FI; ++i)
#pragma unroll
                    for (int j = 0; j < FJ; ++j)
                        sum[i][j] = __builtin_amdgcn_mfma_f32_16x16x4f32(f.b[k][j][r], f.a[k][i][r], sum[i][j], 0, 0, 0);
    };
#pragma unroll
    for (int r = 0; r < AHEAD; ++r) load(ring[r], r);
    store(ring[0], 0);
    load(ring[0], AHEAD);
    if (stages > 1) store(ring[1], 1);
    load(ring[1], AHEAD + 1);
    __syncthreads();
    Fragments f[2];
    read(f[0], 0);
    constexpr int READS = STEPS * (FI * (A_K ? 1 : 4) + FJ * (B_K ? 1 : 4)), PRODUCTS = STEPS * 4 * FI * FJ;
    int t = 0;
    for (; t + 2 * AHEAD + 1 < whole; t += AHEAD)
#pragma unroll
        for (int r = 0; r < AHEAD; ++r) {
            Stage& next = ring[(r + 2) % AHEAD];
            lds_barrier();
            __builtin_amdgcn_sched_barrier(0);
            read(f[(r + 1) & 1], t + r + 1);
            store(next, t + r + 2);
            pa.template load<true>(next.a, 0);
            pb.template load<true>(next.b, 0);
            multiply(f[r & 1]);
            interleave<READS, PRODUCTS / 2, (READS < PRODUCTS / 2 ? READS : PRODUCTS / 2)>();
            __builtin_amdgcn_sched_group_barrier(0x200, 16, 0);
            __builtin_amdgcn_sched_group_barrier(0x020, 16, 0);
            __builtin_amdgcn_sched_group_barrier(0x008, PRODUCTS - PRODUCTS / 2, 0);
            __builtin_amdgcn_sched_barrier(0);
        }
    for (; t < stages; t += AHEAD)
#pragma unroll
        for (int r = 0; r < AHEAD; ++r)
            if (t + r < stages) {
                Stage& next = ring[(r + 2) % AHEAD];
                __syncthreads();
                if (t + r + 1 < stages) read(f[(r + 1) & 1], t + r + 1);
                if (t + r + 2 < stages) store(next, t + r + 2);
                load(next, t + r + 2 + AHEAD);
                multiply(f[r & 1]);
            }

    // the first operand's index is the instruction's row: a lane has columns 4 q .. 4 q + 3 of row lane % 16
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int j = 0; j < FJ; ++j) {
        const int in_col = wj + 16 * j + lane / 16 * 4, col = j0 + in_col;
        float bias[4];
        load_bias(a.e, col, a.J, bias);
        float z[FI][4];
        int64_t row[FI];
#pragma unroll
        for (int i = 0; i < FI; ++i) {
            const int in_row = wi + 16 * i + lane % 16;
            row[i] = i0 + in_row;
#pragma unroll
            for (int r = 0; r < 4; ++r) z[i][r] = sum[i][j][r];
            if (share.splits > 1) store_values(a.partial + (share.slot * TI + in_row) * TJ + in_col, z[i]);
        }
        if (share.splits == 1 && row[0] < a.I && col < a.J) finish<float>(a.e, row, col, a.I, a.J, bias, z);
    }
}

}  // namespace product
}  // namespace lutnn
