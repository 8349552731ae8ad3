// Products of operands as they are, at any address and stride: of fp32 ones on the fp32 matrix instructions, for layers of some
// hundred rows, where laying the planes of dense_product.h out takes longer than their faster products save, and of 16-bit ones
// whose rows are no whole aligned 16-byte units, where laying those out takes as long as the product.
//
// fp32: what bounds it is the instructions, 614 GFLOP/s a compute unit: a 64 x 64 tile by 32 k takes 0.48 us of 0.43.  256 x 768 x
// 768 7.7 us (planes 20; straight from memory 10.7), 1024 x 768 x 768 15 (planes 29), 256 x 2048 x 2048 23 (planes 32); from
// 2048 x 1024 x 1024 (39 and 40) on the planes are faster.  16 bits: what bounds it is the loads, which cost by the lines that they
// touch.  1001 x 515 x 1030 10.4 us (laid out 13.6), 256 x 2047 x 2047 17 (21), 1024 x 767 x 767 10.5 (11.4); 2048 x 2047 x 2047 52
// (36).
// Values go through registers to LDS, two stages ahead of that, so that rows of any alignment are read 16 bytes at a time: four
// stages took 8 % longer, a third of it the first loads, but for a few rows by a W past the caches (64 x 4096 x 4096 in fp32 26 us
// for 34; the sum is shared out there, 25).  A stage's operands are read from LDS while the last one's products run (fp32, 64 x 64:
// 18 % faster than behind its barrier).  Wider tiles leave too few workgroups where this is used; 64 x 32 is no faster than
// 32 x 32 in fp32.
#pragma once
#include <type_traits>

#include "dense_tiles.h"
#include "matrix_types.h"

namespace lutnn {
namespace product {

// 16-byte units of one operand's tile, OUT outer indices by DEPTH k, on their way from memory to LDS through registers.  An
// operand whose rows do not run along k has a unit's values of outer indices at least.
template <class T, int OUT, int DEPTH, bool K_INNER, int THREADS>
struct Panel {
    static constexpr int kUnit = 16 / sizeof(T);
    static constexpr int kLoads = OUT * DEPTH / kUnit / THREADS, kInRow = (K_INNER ? DEPTH : OUT) / kUnit;  // units
    static constexpr int kFront = K_INNER ? 0 : kUnit;  // of a row in LDS
    static constexpr int kPitch = (K_INNER ? DEPTH : OUT) + kUnit, kValues = kPitch * (K_INNER ? OUT : DEPTH);
    static_assert(kLoads * THREADS * kUnit == OUT * DEPTH, "whole loads");
    typedef T Unit __attribute__((ext_vector_type(kUnit)));
    typedef typename Packed<T, kUnit>::type Loose;  // at any address

    const T* at[kLoads];
    int to[kLoads];
    int64_t step;

    __device__ __forceinline__ Panel(const Operand& o, int64_t first, int64_t count, int64_t k0) {
        const T* const p = static_cast<const T*>(o.p);
        step = K_INNER ? DEPTH : DEPTH * o.ld;
#pragma unroll
        for (int l = 0; l < kLoads; ++l) {
            const int u = l * THREADS + threadIdx.x, row = u / kInRow;
            int col = u % kInRow * kUnit;
            if constexpr (K_INNER) {
                at[l] = p + min(first + row, count - 1) * o.ld + k0 + col;
            } else {  // units past the last column are moved back to end with it, repeating others' values, up to a unit
                      // less one column in front of the tile
                col = (int)min((int64_t)col, count - kUnit - first);
                at[l] = p + (k0 + row) * o.ld + first + col;
            }
            to[l] = row * kPitch + kFront + col;
        }
    }

    // left: the values of k from this tile on; what lies behind them becomes zero.
    template <bool WHOLE>
    __device__ __forceinline__ void load(Unit (&v)[kLoads], int left) {
#pragma unroll
        for (int l = 0; l < kLoads; ++l) {
            const int u = l * THREADS + threadIdx.x;
            if constexpr (WHOLE) {
                v[l] = *reinterpret_cast<const Loose*>(at[l]);
            } else if constexpr (K_INNER) {
                const int k = u % kInRow * kUnit;
#pragma unroll
                for (int r = 0; r < kUnit; ++r) v[l][r] = k + r < left ? at[l][r] : (T)0.f;
            } else {
                const int k = u / kInRow;
                v[l] = Unit{};
                if (k < left) v[l] = *reinterpret_cast<const Loose*>(at[l]);
            }
            at[l] += step;
        }
    }

    // MOVED: units of it may have been moved back.
    template <bool MOVED>
    __device__ __forceinline__ void store(const Unit (&v)[kLoads], T* panel) const {
        typedef typename std::conditional<K_INNER || !MOVED, Unit, Loose>::type To;
#pragma unroll
        for (int l = 0; l < kLoads; ++l) *reinterpret_cast<To*>(panel + to[l]) = v[l];
    }

    // A unit's k of 16 outer indices from `first` on, one per lane: those from k + kUnit q on in lane group q.
    static __device__ __forceinline__ auto fragment(const T* panel, int first, int k) {
        const int lane = threadIdx.x & 63, i = lane & 15, from = k + lane / 16 * kUnit;
        typedef typename std::conditional<sizeof(T) == 4, f32x4, s16x8>::type Fragment;
        if constexpr (K_INNER) {
            return *reinterpret_cast<const Fragment*>(panel + (first + i) * kPitch + from);
        } else if constexpr (sizeof(T) == 4) {
            f32x4 v;
#pragma unroll
            for (int r = 0; r < 4; ++r) v[r] = panel[(from + r) * kPitch + kFront + first + i];
            return v;
        } else {
            typedef __attribute__((address_space(3))) s16x4* lds4;
            s16x4 half[2];
#pragma unroll
            for (int h = 0; h < 2; ++h)  // lane i gets column i of the four rows of 16 values that its 16 lanes name
                half[h] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4)(panel + (from + 4 * h + (i >> 2)) * kPitch + kFront + first + (i & 3) * 4));
            return __builtin_shufflevector(half[0], half[1], 0, 1, 2, 3, 4, 5, 6, 7);
        }
    }
};

// As Config of dense_product.h.  WAVES: of a SIMD unit, at least; what the registers have to leave room for.
template <class T_, int TI_, int TJ_, int WI_, int WJ_, int DEPTH_, int WAVES_>
struct ConfigAsIs {
    typedef T_ T;
    static constexpr bool AS_IS = true;
    static constexpr int TI = TI_, TJ = TJ_, WI = WI_, WJ = WJ_, DEPTH = DEPTH_, THREADS = 64 * WI * WJ, WAVES = WAVES_;
    static constexpr int values(int out) { return out * DEPTH + 16 / (int)sizeof(T) * (out > DEPTH ? out : DEPTH); }
    static constexpr int LDS = 2 * (int)sizeof(T) * (values(TI) + values(TJ));
};

// Workgroup `block`'s tile.  Stage t + 1's operands are read from LDS, stage t + 2's written there and stage t + 4's asked for while
// stage t's are multiplied.
template <class C, bool A_K, bool B_K>
__device__ __forceinline__ void tile_as_is(const ProductArgs& a, int block, char* const lds) {
    typedef typename C::T T;
    constexpr bool F32 = sizeof(T) == 4;
    constexpr int TI = C::TI, TJ = C::TJ, DEPTH = C::DEPTH, FI = TI / C::WI / 16, FJ = TJ / C::WJ / 16, AHEAD = 2;
    constexpr int STEP = F32 ? 16 : 32, STEPS = DEPTH / STEP;  // k
    typedef Panel<T, TI, DEPTH, A_K, C::THREADS> PanelA;
    typedef Panel<T, TJ, DEPTH, B_K, C::THREADS> PanelB;
    constexpr int BUF = PanelA::kValues + PanelB::kValues;
    static_assert(2 * BUF * sizeof(T) <= C::LDS, "two buffers");
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
    T* const buffers = reinterpret_cast<T*>(lds);

    struct Stage {
        typename PanelA::Unit a[PanelA::kLoads];
        typename PanelB::Unit b[PanelB::kLoads];
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
    struct Fragments {
        decltype(PanelA::fragment(nullptr, 0, 0)) a[STEPS][FI], b[STEPS][FJ];
    };
    const auto read = [&](Fragments& f, int t) {
        const T *const at = buffers + (t & 1) * BUF, *const bt = at + PanelA::kValues;
#pragma unroll
        for (int k = 0; k < STEPS; ++k) {
#pragma unroll
            for (int i = 0; i < FI; ++i) f.a[k][i] = PanelA::fragment(at, wi + 16 * i, STEP * k);
#pragma unroll
            for (int j = 0; j < FJ; ++j) f.b[k][j] = PanelB::fragment(bt, wj + 16 * j, STEP * k);
        }
    };
    const auto multiply = [&](const Fragments& f) {
#pragma unroll
        for (int k = 0; k < STEPS; ++k)
#pragma unroll
            for (int r = 0; r < (F32 ? 4 : 1); ++r)
#pragma unroll
                for (int i = 0; i < FI; ++i)
#pragma unroll
                    for (int j = 0; j < FJ; ++j)
                        if constexpr (F32)
                            sum[i][j] = __builtin_amdgcn_mfma_f32_16x16x4f32(f.b[k][j][r], f.a[k][i][r], sum[i][j], 0, 0, 0);
                        else
                            sum[i][j] = mfma(f.b[k][j], f.a[k][i], sum[i][j], T());
    };
    const auto run = [&](auto moved) {
        constexpr bool MOVED = decltype(moved)::value;
        const auto store = [&](const Stage& s, int t) {
            T* const to = buffers + (t & 1) * BUF;
            pa.template store<MOVED>(s.a, to);
            pb.template store<MOVED>(s.b, to + PanelA::kValues);
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
        constexpr int TURN = F32 ? 4 : 2;  // LDS reads of a fragment that is turned
        constexpr int READS = STEPS * (FI * (A_K ? 1 : TURN) + FJ * (B_K ? 1 : TURN)), PRODUCTS = STEPS * (F32 ? 4 : 1) * FI * FJ;
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
    };
    // unaligned stores of 16-bit values to LDS go one by one
    if constexpr (F32)
        run(std::true_type());
    else if ((!A_K && i0 + TI > a.I) || (!B_K && j0 + TJ > a.J))
        run(std::true_type());
    else
        run(std::false_type());

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
        if (share.splits == 1 && row[0] < a.I && col < a.J) finish<T>(a.e, row, col, a.I, a.J, bias, z);
    }
}

}  // namespace product
}  // namespace lutnn
