// The matrix products of dense linear layers on the matrix cores, C[i][j] = sum_k A(i, k) B(k, j), with the layer's epilogue: of
// 16-bit operands in whole aligned 16-byte units, and of fp32 ones as three planes of bf16 parts, a = h + m + l, a b being
// l h' + h l' + m m' + m h' + h m' + h h' (split_bf16.h): six products at a sixteenth of the fp32 instructions' cost each.
//
// What bounds them is the matrix instructions, and for the largest the power they draw.  16384 x 4096 x 4096 in bf16, us:
//   X W 395 (1390 TFLOP/s), dZ W^T 402, X^T dZ 393; with the activations of a layer, 16384 x 1024 x 4096, 125, gelu 152, gelu and Z
//   kept 156 (268 MB written in 31).  fp32, both gradients'
//   products of 4096 x 768 x 2304, 160 (181 TFLOP/s, of six products 1090).
// How it gets there, and what was slower:
//   - Tiles of 256 x 256 by eight wavefronts of 128 x 64: every operand is read from LDS once per 128 or 64 products.  Two
//     workgroups of 128 x 256 to a compute unit, so that one's epilogue runs beside the other's products: 419 to 500 us, and no
//     faster at K = 1024.  Instructions of 32 x 32: 425.
//   - Loads go straight to LDS, a ring of three stages of 32 k; two of 64 k 430 and more.  A stage's barrier lets loads fly on.
//   - The next step's operands are read from LDS while a step's products run, a read between every two.
//   - Operands whose rows do not run along k are turned by the LDS reads, so that no layout needs a pass over memory.
//   - XORed units keep those reads from meeting in a bank.  Tiles go to the XCDs in contiguous ranges, four rows of tiles at a time.
// Operands of odd strides or addresses are laid out first, or go through dense_tile_as_is.h.  Which tile, and whether a sum is shared
// out: dense_linear.hip.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "dense_tile_as_is.h"
#include "lutnn_kernels.h"
#include "mfma_tile.h"
#include "split_bf16.h"

namespace lutnn {
namespace product {

typedef int i32x4 __attribute__((ext_vector_type(4)));

constexpr uint32_t kBeyond = 0xc0000000u;  // an offset past any tile's rows: the load gives zeros

// What a wavefront's lanes have written to LDS is there for its other lanes.
__device__ __forceinline__ void wave_sync() {
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

// 64 lanes x 16 bytes from the buffer `rsrc` straight into LDS at lds_dst + 16 * lane; zeros for offsets past its end.  Nothing
// is said of LDS being written: reads of other buffers may move across, and wait_loads keeps those of this one behind it.
__device__ __forceinline__ void buffer_to_lds(uint32_t lds_dst, i32x4 rsrc, uint32_t voff) {
    asm volatile(
        "s_mov_b32 m0, %0\n\t"
        "s_nop 0\n\t"
        "buffer_load_dwordx4 %1, %2, 0 offen lds"
        :
        : "s"(lds_dst), "v"(voff), "s"(rsrc)
        : "m0");
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
    static_assert(K_INNER ? kUnits == 4 || kUnits == 8 : kUnits >= 4, "units to move");

    // Where unit u of a row lies in it.  k inner: rows of 128 or 64 bytes, read 16 of them at a time at one unit; the same unit of
    // eight (four) neighbouring rows lies in different banks.  Otherwise rows k .. k + 3 of each of four groups eight apart are read
    // at once, 32 bytes of each: pairs of units are moved.
    static __device__ __forceinline__ int place(int row, int u) {
        if constexpr (K_INNER) return kUnits == 8 ? u ^ ((row >> 1) & 7) : u ^ ((row >> 1) & 3);
        if constexpr (kUnits >= 16) return u ^ (((row & 3) | ((row >> 1) & 4)) << 1);
        if constexpr (kUnits == 8) return u ^ ((row & 3) << 1);
        return u ^ ((row >> 2) & 2);
    }

    const char* at;          // the next k tile's first value
    int64_t plane, k_step;   // bytes between the parts, and from one k tile to the next
    uint32_t stride, end;    // bytes: of a row, and of a whole k tile's range in memory
    uint32_t off[kLoads];    // of this thread's units
    uint32_t to;             // where a wavefront's units go in a buffer

    __device__ __forceinline__ Tile(const Operand& o, int64_t first, int64_t count, int64_t k0) {
        stride = (uint32_t)(o.ld * 2);
        plane = o.plane * 2;
        if constexpr (K_INNER) {
            at = static_cast<const char*>(o.p) + (first * o.ld + k0) * 2;
            k_step = DEPTH * 2;
            end = (uint32_t)(min((int64_t)OUT, count - first) - 1) * stride + DEPTH * 2;
        } else {
            at = static_cast<const char*>(o.p) + (k0 * o.ld + first) * 2;
            k_step = (int64_t)DEPTH * stride;
            end = (DEPTH - 1) * stride + (uint32_t)(min((int64_t)OUT, (count - first + 7) / 8 * 8) * 2);
        }
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            const int slot = i * THREADS + threadIdx.x, row = slot / kUnits;
            off[i] = (uint32_t)row * stride + (uint32_t)place(row, slot % kUnits) * 16;
        }
        to = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) * 1024;
    }

    // Loads the next k tile into LDS at `buffer`.  left: the values of k from there on; DEPTH or more for a whole tile.
    template <bool WHOLE>
    __device__ __forceinline__ void load(uint32_t buffer, int left) {
        uint32_t size = end;
        // rows that run along k end in zeros as far as their last unit goes; what lies behind is not theirs
        if constexpr (!WHOLE) size -= K_INNER ? (uint32_t)(DEPTH - (left + 7) / 8 * 8) * 2 : (uint32_t)(DEPTH - left) * stride;
#pragma unroll
        for (int p = 0; p < PARTS; ++p) {
            const uint64_t from = reinterpret_cast<uint64_t>(at + p * plane);
            const i32x4 rsrc = {(int)(uint32_t)from, (int)(uint32_t)(from >> 32), (int)size, 0x00020000};
#pragma unroll
            for (int i = 0; i < kLoads; ++i) {
                uint32_t o = off[i];
                if constexpr (!WHOLE && K_INNER) {
                    const int slot = i * THREADS + threadIdx.x, row = slot / kUnits;
                    if (place(row, slot % kUnits) * 8 >= left) o = kBeyond;
                }
                buffer_to_lds(buffer + to + p * kPart + i * THREADS * 16, rsrc, o);
            }
        }
        at += k_step;
    }

    // The matrix instruction's operand: 16 outer indices from `first` on, one per lane, by the s-th 32 k, eight per lane.
    static __device__ __forceinline__ s16x8 fragment(const char* part, int first, int s) {
        const int lane = threadIdx.x & 63, i = lane & 15, q = lane >> 4;
        if constexpr (K_INNER) {
            const int row = first + i;
            return *reinterpret_cast<const s16x8*>(part + row * kRow * 2 + place(row, 4 * s + q) * 16);
        } else {
            typedef __attribute__((address_space(3))) s16x4* lds4;
            s16x4 half[2];
#pragma unroll
            for (int h = 0; h < 2; ++h) {  // lane i gets column i of the four rows of 16 values that its 16 lanes name
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

// A tile's size, wavefronts and ring.  T: the matrices' type; fp32 ones are three planes of bf16 (split_bf16.h).
template <class T_, int TI_, int TJ_, int WI_, int WJ_, int DEPTH_, int STAGES_>
struct Config {
    typedef T_ T;
    static constexpr bool F32 = sizeof(T) == 4, AS_IS = false;
    static constexpr int TI = TI_, TJ = TJ_, WI = WI_, WJ = WJ_, DEPTH = DEPTH_, STAGES = STAGES_;
    static constexpr int PARTS = F32 ? 3 : 1, THREADS = 64 * WI * WJ, WAVES = 2, BUF = (TI + TJ) * DEPTH * 2 * PARTS;
    // the sums on their way out: a wavefront's, ROUND rows at a time
    static constexpr int ROUND = TI / WI < 64 ? TI / WI : 64, COLS = TJ / WJ, PITCH = COLS + 4, OUT = WI * WJ * ROUND * PITCH * 4;
    static constexpr int LDS = STAGES * BUF > OUT ? STAGES * BUF : OUT;
};

// Workgroup `block`'s tile of a product; lds: C::LDS bytes.
template <class C, bool A_K, bool B_K>
__device__ __forceinline__ void product_tile(const ProductArgs& a, int block, char* const lds) {
    typedef typename C::T T;
    constexpr bool F32 = C::F32;
    constexpr int PARTS = C::PARTS, THREADS = C::THREADS, DEPTH = C::DEPTH, STAGES = C::STAGES, TI = C::TI, TJ = C::TJ, WI = C::WI, WJ = C::WJ;
    constexpr int FI = TI / WI / 16, FJ = TJ / WJ / 16, STEPS = DEPTH / 32, BUF = C::BUF;
    constexpr int ROUND = C::ROUND, COLS = C::COLS, PITCH = C::PITCH, kBatch = TI * TJ > 128 * 128 ? 4 : 2;
    typedef typename std::conditional<F32, bf16, T>::type E;
    typedef Tile<TI, DEPTH, A_K, PARTS, THREADS> TileA;
    typedef Tile<TJ, DEPTH, B_K, PARTS, THREADS> TileB;
    static_assert(BUF == TileA::kBytes + TileB::kBytes, "a stage's operands");

    const Share share = share_of(a, block);
    if (share.tile < 0) return;
    const int splits = share.splits, split = share.split;
    const TilePlace at = place_of(share.tile, a.i_tiles, a.j_tiles);
    const int64_t i0 = (int64_t)at.i * TI;
    const int j0 = at.j * TJ;

    const int k_tiles = (int)((a.K + DEPTH - 1) / DEPTH);
    const int t0 = (int)((int64_t)k_tiles * split / splits), stages = (int)((int64_t)k_tiles * (split + 1) / splits) - t0;
    const int k_left = (int)min(a.K - (int64_t)t0 * DEPTH, (int64_t)stages * DEPTH), whole = k_left / DEPTH;
    TileA ta(a.A, i0, a.I, (int64_t)t0 * DEPTH);
    TileB tb(a.B, j0, a.J, (int64_t)t0 * DEPTH);

    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wi = wave / WJ * (TI / WI), wj = wave % WJ * (TJ / WJ);
    f32x4 sum[FI][FJ] = {};
    struct Fragments {
        s16x8 a[F32 ? 1 : FI], b[PARTS][FJ];
    };
    const auto read_a = [&](s16x8& f, int buffer, int p, int i, int s) {
        f = TileA::fragment(lds + buffer * BUF + p * TileA::kPart, wi + 16 * i, s);
    };
    const auto read_b = [&](Fragments& f, int buffer, int s) {
#pragma unroll
        for (int p = 0; p < PARTS; ++p)
#pragma unroll
            for (int j = 0; j < FJ; ++j)
                f.b[p][j] = TileB::fragment(lds + buffer * BUF + TileA::kBytes + p * TileB::kPart, wj + 16 * j, s);
    };

    // A ring of STAGES buffers, one k tile each.  While a step's products run from registers, the next step's operands are read:
    // a stage's barrier says that the next one has arrived and that everybody has read all of this one, whose buffer is loaded anew.
    const uint32_t base = lds_offset(lds);
    constexpr int LOADS = PARTS * (TileA::kLoads + TileB::kLoads);
    const auto load = [&](int buffer, int t) {
        if (t < whole) {
            ta.template load<true>(base + buffer * BUF, 0);
            tb.template load<true>(base + buffer * BUF + TileA::kBytes, 0);
        } else {
            ta.template load<false>(base + buffer * BUF, k_left - t * DEPTH);
            tb.template load<false>(base + buffer * BUF + TileA::kBytes, k_left - t * DEPTH);
        }
    };
#pragma unroll 1
    for (int i = 0; i < STAGES; ++i)
        if (i < stages) load(i, i);
    if (STAGES <= stages)
        wait_loads<(STAGES - 1) * LOADS>();
    else
        wait_loads<0>();
    lds_barrier();
    Fragments now, then;
    int buffer = 0;
    // On to stage t + 1: its buffer, and stage t's to load into.
    const auto arrive = [&](int t, auto steady) {
        const int from = buffer;
        buffer = buffer + 1 == STAGES ? 0 : buffer + 1;
        if (decltype(steady)::value || t + STAGES <= stages)
            wait_loads<(STAGES - 2) * LOADS>();
        else
            wait_loads<0>();
        lds_barrier();
        return from;
    };
    const auto refill = [&](int from, int t, auto steady) {
        if constexpr (decltype(steady)::value) {
            ta.template load<true>(base + from * BUF, 0);
            tb.template load<true>(base + from * BUF + TileA::kBytes, 0);
        } else if (t + STAGES < stages) {
            load(from, t + STAGES);
        }
    };
    constexpr int READ_A = A_K ? 1 : 2, READ_B = B_K ? 1 : 2;  // instructions per fragment
    constexpr int PAIR = 2 / STEPS;                            // stages of two steps
    static_assert(STEPS <= 2, "steps of a stage");
    const auto run = [&](auto&& step) {
        int t = 0;
        for (; t + PAIR - 1 + STAGES < whole; t += PAIR) {
            step(now, then, t, 0, std::true_type());
            step(then, now, t + PAIR - 1, STEPS - 1, std::true_type());
        }
        for (; t + PAIR <= stages; t += PAIR) {
            step(now, then, t, 0, std::false_type());
            step(then, now, t + PAIR - 1, STEPS - 1, std::false_type());
        }
        if (t < stages) step(now, then, t, 0, std::false_type());
    };
    read_b(now, 0, 0);
    if constexpr (!F32) {
        const auto read_all_a = [&](Fragments& f, int s) {
#pragma unroll
            for (int i = 0; i < FI; ++i) read_a(f.a[i], buffer, 0, i, s);
        };
        read_all_a(now, 0);
        run([&](const Fragments& f, Fragments& next, int t, int s, auto steady) {
            const bool last = s + 1 == STEPS;
            int from = 0;
            if (last) {
                from = arrive(t, steady);
                if constexpr (!decltype(steady)::value) refill(from, t, steady);
            }
            read_b(next, buffer, last ? 0 : s + 1);  // behind the last stage: something, unused
            read_all_a(next, last ? 0 : s + 1);
            if constexpr (decltype(steady)::value)
                if (last) refill(from, t, steady);
#pragma unroll
            for (int i = 0; i < FI; ++i)
#pragma unroll
                for (int j = 0; j < FJ; ++j) sum[i][j] = mfma(f.b[0][j], f.a[i], sum[i][j], E());
            interleave<FI * READ_A + FJ * READ_B, FI * FJ, FI * FJ / 2>();
            __builtin_amdgcn_sched_barrier(0);
        });
    } else {
        // A's fragments are read one row of them ahead, B's one stage: the last row's products hide those.
        static_assert(STEPS == 1 && FI % 2 == 0, "two rows in turn");
        s16x8 row[2][3];
        const auto read_row = [&](int i) {
#pragma unroll
            for (int p = 0; p < 3; ++p) read_a(row[i & 1][p], buffer, p, i % FI, 0);
        };
        read_row(0);
        run([&](const Fragments& f, Fragments& next, int t, int, auto steady) {
#pragma unroll
            for (int i = 0; i < FI; ++i) {
                if (i + 1 == FI) {
                    const int from = arrive(t, steady);
                    if constexpr (!decltype(steady)::value) refill(from, t, steady);
                    read_b(next, buffer, 0);
                    read_row(FI);
                    if constexpr (decltype(steady)::value) refill(from, t, steady);
                } else {
                    read_row(i + 1);
                }
                constexpr int kPairs[6][2] = {{2, 0}, {0, 2}, {1, 1}, {1, 0}, {0, 1}, {0, 0}};  // small products first
                f32x4 slice[FJ] = {};
#pragma unroll
                for (int n = 0; n < 6; ++n)
#pragma unroll
                    for (int j = 0; j < FJ; ++j) slice[j] = mfma(f.b[kPairs[n][1]][j], row[i & 1][kPairs[n][0]], slice[j], E());
#pragma unroll
                for (int j = 0; j < FJ; ++j) sum[i][j] += slice[j];
                if (i + 1 == FI)
                    interleave<3 * (READ_A + FJ * READ_B), 6 * FJ, 3 * FJ>();
                else
                    interleave<3 * READ_A, 3 * FJ, 3>();
                __builtin_amdgcn_sched_barrier(0);
            }
        });
    }
    wait_loads<0>();

    // Out through LDS, so that a row's values leave in whole lines: every wavefront its own, nothing to wait for but that all
    // have read their operands.
    constexpr int VEC = F32 ? 4 : 8, LANES = COLS / VEC, STEP = 64 / LANES;  // values per lane, lanes per row, rows at once
    constexpr int BATCH = ROUND / STEP < kBatch ? ROUND / STEP : kBatch;
    const int lane = threadIdx.x & 63;
    const int in_cols = wj + lane % LANES * VEC, col = j0 + in_cols;
    float bias[VEC];
    load_bias(a.e, col, a.J, bias);
    // A residual without an activation, in whole units: a round's rows are asked for at once and a round ahead, into registers that
    // held operands and sums.  Batch by batch each would wait for its own.
    constexpr int PER = ROUND / STEP, ROUNDS = TI / WI / ROUND;
    const bool added = splits == 1 && a.e.R && a.e.activation == kActNone && !a.e.Z && col + VEC <= a.J;
    typename Packed<T, VEC>::type residual[ROUNDS][PER];
    const auto fetch = [&](int round) {
        if (!added) return;
#pragma unroll
        for (int r = 0; r < PER; ++r) {
            const int64_t row = min(i0 + wi + round * ROUND + r * STEP + lane / LANES, a.I - 1);
            residual[round][r] = *reinterpret_cast<const typename Packed<T, VEC>::type*>(static_cast<const T*>(a.e.R) + row * a.e.ldr + col);
        }
    };
    fetch(0);
    lds_barrier();
    float* const out = reinterpret_cast<float*>(lds) + wave * ROUND * PITCH;
#pragma unroll
    for (int round = 0; round < ROUNDS; ++round) {
        float probe = 0.f;
        if (round > 0) wave_sync();  // the last round has been read
#pragma unroll
        for (int i = 0; i < ROUND / 16; ++i)
#pragma unroll
            for (int j = 0; j < FJ; ++j) {  // a lane has four columns of a row
                f32x4 z = sum[round * ROUND / 16 + i][j];
                if constexpr (F32) {
                    z *= kUnscale;
                    probe += fabsf(z[0]) + fabsf(z[1]) + (fabsf(z[2]) + fabsf(z[3]));
                }
                *reinterpret_cast<f32x4*>(out + (16 * i + lane % 16) * PITCH + 16 * j + 4 * (lane / 16)) = z;
            }
        wave_sync();
        if constexpr (F32)
            // sums that are not finite are formed again: an infinite value has no parts
            if (splits == 1 && __any(!is_finite(probe))) {
#pragma unroll 1
                for (int v = lane; v < ROUND * COLS; v += 64) {
                    const int64_t i = i0 + wi + round * ROUND + v / COLS;
                    const int j = j0 + wj + v % COLS;
                    float& z = out[v / COLS * PITCH + v % COLS];
                    if (i < a.I && j < a.J && !is_finite(z)) z = chain(a, i, j);
                }
                wave_sync();
            }
        if (round + 1 < ROUNDS) fetch(round + 1);
        if (added) {
#pragma unroll
            for (int r = 0; r < PER; ++r) {
                float z[VEC];
                load_values(out + (r * STEP + lane / LANES) * PITCH + lane % LANES * VEC, z);
#pragma unroll
                for (int c = 0; c < VEC; ++c) z[c] += bias[c] + (float)residual[round][r][c];
                const int64_t row = i0 + wi + round * ROUND + r * STEP + lane / LANES;
                if (row < a.I) store_values(static_cast<T*>(a.e.Y) + row * a.e.ldy + col, z);
            }
            continue;
        }
#pragma unroll 1
        for (int b = 0; b < PER; b += BATCH) {
            float z[BATCH][VEC];
            int64_t row[BATCH];
            const int first = b * STEP + lane / LANES, in_rows = wi + round * ROUND + first;
#pragma unroll
            for (int r = 0; r < BATCH; ++r) {
                load_values(out + (first + r * STEP) * PITCH + lane % LANES * VEC, z[r]);
                row[r] = i0 + in_rows + r * STEP;
            }
            if (splits > 1) {
                float* const to = a.partial + (share.slot * TI + in_rows) * TJ + in_cols;
#pragma unroll
                for (int r = 0; r < BATCH; ++r) store_values(to + r * STEP * TJ, z[r]);
                continue;
            }
            if (row[0] >= a.I || col >= a.J) continue;
            finish<T>(a.e, row, col, a.I, a.J, bias, z);
        }
    }
}

template <class C, bool A_K, bool B_K>
__device__ __forceinline__ void any_tile(const ProductArgs& a, int block, char* const lds) {
    if constexpr (C::AS_IS)
        tile_as_is<C, A_K, B_K>(a, block, lds);
    else
        product_tile<C, A_K, B_K>(a, block, lds);
}

template <class C, bool A_K, bool B_K>
__global__ __launch_bounds__(C::THREADS, C::WAVES) void product_kernel(ProductArgs a) {
    __shared__ __align__(1024) char lds[C::LDS];
    any_tile<C, A_K, B_K>(a, blockIdx.x, lds);
}

// dX = dZ W^T and dW = X^T dZ in one launch, that with the longer tiles first, and db's partial sums added up beside them.
template <class C>
__global__ __launch_bounds__(C::THREADS, C::WAVES) void pair_kernel(PairArgs p) {
    __shared__ __align__(1024) char lds[C::LDS];
    const int first = p.x_first ? p.x_blocks : p.w_blocks, both = p.x_blocks + p.w_blocks, b = blockIdx.x;
    if (b >= both)
        add_partial_sums<typename C::T, C::THREADS>(p.sums, b - both, lds);
    else if ((b < first) == (p.x_first != 0))
        any_tile<C, true, true>(p.x, b < first ? b : b - first, lds);
    else
        any_tile<C, false, false>(p.w, b < first ? b : b - first, lds);
}

// The shared tiles' sums through the epilogue, four columns per thread.  TI x TJ: a tile.
template <class T, int TI, int TJ>
__global__ __launch_bounds__(256) void join_kernel(ProductArgs a) {
    constexpr int QUADS = TI * TJ / 4;
    const int shared = a.i_tiles * a.j_tiles - a.whole;
    for (int64_t v = blockIdx.x * 256LL + threadIdx.x; v < (int64_t)shared * QUADS; v += gridDim.x * 256LL) {
        const int tile = (int)(v / QUADS), in_tile = (int)(v % QUADS) * 4;
        const TilePlace at = place_of(a.whole + tile, a.i_tiles, a.j_tiles);
        const int64_t i = (int64_t)at.i * TI + in_tile / TJ;
        const int j = at.j * TJ + in_tile % TJ;
        if (i >= a.I || j >= a.J) continue;
        const float* from = a.partial + (int64_t)tile * TI * TJ + in_tile;
        float z[4] = {};
        for (int s = 0; s < a.splits; ++s, from += (int64_t)shared * TI * TJ) {
            float x[4];
            load_values(from, x);
#pragma unroll
            for (int r = 0; r < 4; ++r) z[r] += x[r];
        }
        if constexpr (sizeof(T) == 4)
            for (int r = 0; r < 4 && j + r < a.J; ++r)
                if (!is_finite(z[r])) z[r] = chain(a, i, j + r);
        float bias[4], rows[1][4] = {{z[0], z[1], z[2], z[3]}};
        load_bias(a.e, j, a.J, bias);
        const int64_t row[1] = {i};
        finish<T>(a.e, row, j, a.I, a.J, bias, rows);
    }
}

inline unsigned blocks_of(const ProductArgs& a) {
    const int shared = a.i_tiles * a.j_tiles - a.whole;
    return (a.whole + 7) / 8 * 8 + (shared * a.splits + 7) / 8 * 8;
}

// Sets i_tiles and j_tiles; false for too many.
template <class C>
bool count_tiles(ProductArgs& a) {
    const int64_t i_tiles = (a.I + C::TI - 1) / C::TI, j_tiles = (a.J + C::TJ - 1) / C::TJ, tiles = i_tiles * j_tiles;
    if (tiles > kMostTiles || (tiles - a.whole) * a.splits > kMostTiles) return false;
    a.i_tiles = (int)i_tiles, a.j_tiles = (int)j_tiles;
    return true;
}

template <class C>
hipError_t join(const ProductArgs& a, hipStream_t s) {
    const int64_t shared = a.i_tiles * a.j_tiles - a.whole, quads = shared * C::TI * C::TJ / 4;
    if (shared == 0 || a.splits == 1) return hipSuccess;
    hipLaunchKernelGGL((join_kernel<typename C::T, C::TI, C::TJ>), dim3((unsigned)std::min<int64_t>((quads + 255) / 256, 1 << 16)), dim3(256),
                       0, s, a);
    return hipGetLastError();
}

// a.whole: how many tiles not to share.  A's k is inner but for dW = X^T dZ, B's for dX = dZ W^T.
template <class C>
hipError_t launch(ProductArgs a, bool a_k, bool b_k, hipStream_t s) {
    if (!count_tiles<C>(a)) return hipErrorInvalidConfiguration;
    const dim3 grid(blocks_of(a)), threads(C::THREADS);
    if (!a_k)
        hipLaunchKernelGGL((product_kernel<C, false, false>), grid, threads, 0, s, a);
    else if (b_k)
        hipLaunchKernelGGL((product_kernel<C, true, true>), grid, threads, 0, s, a);
    else
        hipLaunchKernelGGL((product_kernel<C, true, false>), grid, threads, 0, s, a);
    if (hipError_t e = hipGetLastError()) return e;
    return join<C>(a, s);
}

template <class C>
hipError_t launch_pair(PairArgs p, hipStream_t s) {
    if (!count_tiles<C>(p.x) || !count_tiles<C>(p.w)) return hipErrorInvalidConfiguration;
    p.x_blocks = (int)blocks_of(p.x), p.w_blocks = (int)blocks_of(p.w);
    const unsigned blocks = p.x_blocks + p.w_blocks + (p.sums.out ? (p.sums.width + 31) / 32 : 0);
    hipLaunchKernelGGL(pair_kernel<C>, dim3(blocks), dim3(C::THREADS), 0, s, p);
    if (hipError_t e = hipGetLastError()) return e;
    if (hipError_t e = join<C>(p.x, s)) return e;
    return join<C>(p.w, s);
}

// Calls f with the Config of a tile of dense_linear.hip's lists.
template <class T, class F>
hipError_t with_tile(int tile, F&& f) {
    if constexpr (sizeof(T) == 4) {
        switch (tile) {
            case 0: return f(Config<T, 128, 256, 2, 4, 32, 2>());
            case 1: return f(Config<T, 128, 128, 2, 4, 32, 2>());
            case 2: return f(ConfigAsIs<T, 64, 64, 2, 4, 32, 4>());
            default: return f(ConfigAsIs<T, 32, 32, 2, 2, 32, 4>());
        }
    } else {
        switch (tile) {
            case 0: return f(Config<T, 256, 256, 2, 4, 32, 3>());
            case 1: return f(Config<T, 128, 128, 2, 4, 64, 2>());
            case 2: return f(Config<T, 64, 128, 2, 4, 64, 2>());
            case 3: return f(Config<T, 64, 64, 2, 2, 64, 3>());
            case 4: return f(Config<T, 32, 64, 1, 4, 64, 3>());
            case 5: return f(ConfigAsIs<T, 64, 64, 2, 2, 64, 2>());
            default: return f(ConfigAsIs<T, 32, 64, 1, 4, 64, 2>());
        }
    }
}

template <class T>
hipError_t launch_tile(int tile, bool a_k, bool b_k, const ProductArgs& a, hipStream_t s) {
    return with_tile<T>(tile, [&](auto c) { return launch<decltype(c)>(a, a_k, b_k, s); });
}
template <class T>
hipError_t launch_tiles(int tile, const PairArgs& p, hipStream_t s) {
    return with_tile<T>(tile, [&](auto c) { return launch_pair<decltype(c)>(p, s); });
}

}  // namespace product

// dense_product_f32.hip, _bf16.hip, _f16.hip
hipError_t launch_product_f32(int tile, bool a_k, bool b_k, const ProductArgs& a, hipStream_t s);
hipError_t launch_product_bf16(int tile, bool a_k, bool b_k, const ProductArgs& a, hipStream_t s);
hipError_t launch_product_f16(int tile, bool a_k, bool b_k, const ProductArgs& a, hipStream_t s);
hipError_t launch_pair_f32(int tile, const PairArgs& p, hipStream_t s);
hipError_t launch_pair_bf16(int tile, const PairArgs& p, hipStream_t s);
hipError_t launch_pair_f16(int tile, const PairArgs& p, hipStream_t s);

}  // namespace lutnn
