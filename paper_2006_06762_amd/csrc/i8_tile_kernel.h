// Products of 8-bit integers in tiles on the matrix pipes (i8_device.h).
//
// A work-group takes a tile of BM x BN, its waves WM x WN parts of it in blocks of 32 x 32 (v_mfma_i32_32x32x32_i8), and walks k in chunks of 128:
// global -> registers -> LDS -> operands, with two LDS buffers, so that one is multiplied while the other is filled and the loads of the chunk
// after that are on their way.
//
// LDS: 128 bytes of k per row, 16-byte units exchanged by pairs of rows (unit ^ row / 2 % 8): two rows fill the 64 banks, and sixteen rows' same
// unit, which an operand read takes together, lie in different ones.
//
// W is the instruction's first operand: register r of a lane is then n = 8 (r / 4) + 4 (lane / 32) + r % 4 of the block and m = lane % 32: four
// neighbouring columns of a row of D.
#pragma once
#include "i8_device.h"

namespace anr {
namespace i8 {

constexpr int kRow = BK;                        // bytes of a row in LDS
template <int BM, int BN>
constexpr size_t lds_bytes() { return 2 * (size_t)(BM + BN) * kRow; }

// The units of a chunk in three parts.
constexpr int part_of(int units, int part) { return (units * part + 2) / 3; }

// Global -> registers -> LDS of R rows of one operand by NT threads.
template <int R, int NT, bool WHOLE, bool CLEAR>
struct Stager {
    static constexpr int UNITS = R * (BK / kUnit) / NT;
    static_assert(R * (BK / kUnit) % NT == 0 && NT % 8 == 0, "whole units for every thread");
    const int8_t* base;             // of the tile's first row
    int K, first, unit;             // this thread's row in the first unit, its unit in the row
    uint32_t offset[UNITS];         // bytes of a row's start from the base
    u32x4 data[UNITS];

    __device__ __forceinline__ void init(const int8_t* p, int64_t ld, int row0, int rows, int k, int tid)
    {
        base = p + row0 * ld;
        K = k;
        first = tid / 8;
        unit = tid % 8;
#pragma unroll
        for (int i = 0; i < UNITS; ++i) offset[i] = (uint32_t)(min(first + i * (NT / 8), rows - row0 - 1) * ld);
    }
    // units FIRST to LAST - 1 of the chunk of k from k0 on; one that lies past K has zeros (WHOLE) or something
    template <int FIRST, int LAST>
    __device__ __forceinline__ void load(int k0)
    {
        const int k = k0 + unit * kUnit;
#pragma unroll
        for (int i = FIRST; i < LAST; ++i) {
            if (WHOLE) {
                const __amdgpu_buffer_rsrc_t rsrc = __builtin_amdgcn_make_buffer_rsrc(const_cast<int8_t*>(base), 0, kExtent, 0x00020000);
                data[i] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(rsrc, (int)(k < K ? offset[i] + k : kNowhere), 0, 0));
            } else {
                data[i] = load_loose(base + offset[i] + loose_start(k, K));
            }
        }
    }
    template <int FIRST, int LAST>
    __device__ __forceinline__ void store(char* lds, int k0)
    {
        if (CLEAR && !WHOLE && k0 + BK > K) {
#pragma unroll
            for (int i = FIRST; i < LAST; ++i) clear_counted(data[i], k0 + unit * kUnit, K);
        }
#pragma unroll
        for (int i = FIRST; i < LAST; ++i) {
            const int r = first + i * (NT / 8);
            *reinterpret_cast<u32x4*>(lds + r * kRow + ((unit ^ ((r >> 1) & 7)) * 16)) = data[i];
        }
    }
};

// Sixteen k from 32 step + 16 (lane / 32) on of row `row0 + lane % 32`.
__device__ __forceinline__ i32x4 operand(const char* lds, int row0, int step, int lane)
{
    const int r = row0 + (lane & 31), u = 2 * step + (lane >> 5);
    return *reinterpret_cast<const i32x4*>(lds + r * kRow + ((u ^ ((r >> 1) & 7)) * 16));
}

// Eight neighbouring elements of a row, of which `in` exist.
template <typename T>
__device__ __forceinline__ void store8(T* p, const float (&v)[8], int in, bool aligned)
{
    if (aligned && in >= 8) {
        store_floats<T, 8>(p, v);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < in) p[i] = from_float<T>(v[i]);
    }
}

// G groups of waves take a tile's chunks in turn, each with buffers and sums of its own, and join the sums in LDS: for products with about as many
// tiles as CUs, whose work-groups are alone on theirs.  T: D's type; int for sums that go to `parts`.
template <typename T, int BM, int BN, int WM, int WN, int G, bool WHOLE>
__global__ __launch_bounds__(64 * WM * WN * G, 64 * WM * WN * G / 256) void tile_kernel(const Args args)
{
    constexpr bool PARTIAL = std::is_same_v<T, int>;
    constexpr int NT = 64 * WM * WN, MB = BM / (32 * WM), NB = BN / (32 * WN);
    constexpr int XBYTES = BM * kRow, BUF = XBYTES + BN * kRow;
    extern __shared__ __attribute__((aligned(16))) char shared[];
    const int group = G > 1 ? __builtin_amdgcn_readfirstlane(threadIdx.x / NT) : 0;
    char* const lds = shared + group * 2 * BUF;
    const int tid = threadIdx.x % NT, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wm = wave / WN, wn = wave % WN;

    // Work-group ids are dealt round-robin over the 8 XCDs, each with its own L2: every XCD gets a contiguous run of tiles,
    // walked in bands of `band` rows of tiles, column by column
    int id = blockIdx.x;
    {
        const int all = (int)gridDim.x, per = all >> 3, rest = all & 7, xcd = id & 7, slot = id >> 3;
        id = xcd * per + (xcd < rest ? xcd : rest) + slot;
    }
    const int split = PARTIAL ? id % args.splits : 0;
    if (PARTIAL) id /= args.splits;
    const int band = id / (args.band * args.tiles_n), rows = min(args.band, args.tiles_m - band * args.band), in_band = id - band * args.band * args.tiles_n;
    const int m0 = (band * args.band + in_band % rows) * BM, n0 = (in_band / rows) * BN;
    const int M = args.M, N = args.N, K = args.K;

    Stager<BM, NT, WHOLE, true> sx;
    Stager<BN, NT, WHOLE, false> sw;
    sx.init(args.x, args.ldx, m0, M, K, tid);
    sw.init(args.w, args.ldw, n0, N, K, tid);
    const int chunks = (K + BK - 1) / BK;
    const int c0 = PARTIAL ? (int)((int64_t)chunks * split / args.splits) : 0, c1 = PARTIAL ? (int)((int64_t)chunks * (split + 1) / args.splits) : chunks;

    // Chunks past the last one load zeros or what is not used: no branch in the loop
    using SX = decltype(sx);
    using SW = decltype(sw);
    auto k_of = [&](int c) { return G > 1 && c >= c1 ? (chunks + 1) * BK : c * BK; };
    auto load = [&](int c, auto part) {
        constexpr int P = decltype(part)::value;
        sx.template load<part_of(SX::UNITS, P), part_of(SX::UNITS, P + 1)>(k_of(c));
        sw.template load<part_of(SW::UNITS, P), part_of(SW::UNITS, P + 1)>(k_of(c));
    };
    auto store = [&](int buf, int c, auto part) {
        constexpr int P = decltype(part)::value;
        sx.template store<part_of(SX::UNITS, P), part_of(SX::UNITS, P + 1)>(lds + buf * BUF, k_of(c));
        sw.template store<part_of(SW::UNITS, P), part_of(SW::UNITS, P + 1)>(lds + buf * BUF + XBYTES, k_of(c));
    };
    using P0 = std::integral_constant<int, 0>;
    using P1 = std::integral_constant<int, 1>;
    using P2 = std::integral_constant<int, 2>;

    i32x16 acc[NB][MB];
#pragma unroll
    for (int n = 0; n < NB; ++n)
#pragma unroll
        for (int m = 0; m < MB; ++m)
#pragma unroll
            for (int r = 0; r < 16; ++r) acc[n][m][r] = 0;

    // A chunk has four steps of 32 k.  The operands of a step are read from LDS while the one before it is multiplied; the next
    // chunk's units go to the other buffer in the first three steps, each followed by the load of the unit of the chunk after that, and
    // the barrier comes before the fourth, in which the first operands of the next chunk are read.
    i32x4 xv[2][MB], wv[2][NB];
    auto operands = [&](int set, int buf, int s) {
        const char* const x = lds + buf * BUF;
#pragma unroll
        for (int n = 0; n < NB; ++n) wv[set][n] = operand(x + XBYTES, (wn * NB + n) * 32, s, lane);
#pragma unroll
        for (int m = 0; m < MB; ++m) xv[set][m] = operand(x, (wm * MB + m) * 32, s, lane);
    };
    auto multiply = [&](int set) {
#pragma unroll
        for (int n = 0; n < NB; ++n)
#pragma unroll
            for (int m = 0; m < MB; ++m) acc[n][m] = __builtin_amdgcn_mfma_i32_32x32x32_i8(wv[set][n], xv[set][m], acc[n][m], 0, 0, 0);
    };
    // what goes between the matrix instructions of a step: the reads of operands, then `units` stores and loads
    auto interleave = [&](auto units_c) {
        constexpr int units = decltype(units_c)::value, kReads = MB + NB, all_ops = kReads + 2 * units, N_ = MB * NB;
        int done = 0;
#pragma unroll
        for (int i = 0; i < N_; ++i) {
            __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
#pragma unroll
            for (; done < (i + 1) * all_ops / N_; ++done) {
                if (done < kReads) __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
                else if ((done - kReads) % 2 == 0) __builtin_amdgcn_sched_group_barrier(0x200, 1, 0);
                else __builtin_amdgcn_sched_group_barrier(0x020, 1, 0);
            }
        }
    };
    const int first = c0 + group, rounds = (c1 - c0 + G - 1) / G;
    load(first, P0{});
    load(first, P1{});
    load(first, P2{});
    store(0, first, P0{});
    store(0, first, P1{});
    store(0, first, P2{});
    load(first + G, P0{});
    load(first + G, P1{});
    load(first + G, P2{});
    __syncthreads();
    operands(0, 0, 0);
#pragma unroll 1
    for (int r = 0; r < rounds; ++r) {
        const int buf = r & 1, c = first + r * G;
        auto step = [&](auto part) {
            constexpr int S = decltype(part)::value;
            operands((S + 1) & 1, buf, S + 1);
            multiply(S & 1);
            store(buf ^ 1, c + G, part);
            load(c + 2 * G, part);
            interleave(std::integral_constant<int, part_of(SX::UNITS, S + 1) - part_of(SX::UNITS, S) + part_of(SW::UNITS, S + 1) - part_of(SW::UNITS, S)>{});
            __builtin_amdgcn_sched_barrier(0);
        };
        step(P0{});
        step(P1{});
        step(P2{});
        __syncthreads();
        operands(0, buf ^ 1, 0);
        multiply(1);
        interleave(std::integral_constant<int, 0>{});
        __builtin_amdgcn_sched_barrier(0);
    }
    __syncthreads();
    if constexpr (G > 1) {
        static_assert(G == 2 && (size_t)BM * BN * 4 <= 2 * G * (size_t)BUF, "the sums of one group fit the chunks' room");
        i32x16* const other = reinterpret_cast<i32x16*>(shared) + (wave * NB * MB) * 64 + lane;
        if (group == 1) {
#pragma unroll
            for (int i = 0; i < NB * MB; ++i) other[i * 64] = acc[i / MB][i % MB];
        }
        __syncthreads();
        if (group == 0) {
#pragma unroll
            for (int i = 0; i < NB * MB; ++i) acc[i / MB][i % MB] += other[i * 64];
        }
        __syncthreads();
        if (group == 1) return;
    }

    // The sums leave through LDS, 32 rows of a wave at a time, so that neighbouring lanes write neighbouring units of a row
    constexpr int ROW = NB * 128 + 16;                                // bytes; the 16 put eight rows' same column in different banks
    static_assert((size_t)(NT / 64) * 32 * ROW <= 2 * (size_t)BUF, "fits the chunks' room");
    char* const own = lds + wave * 32 * ROW;
    constexpr int LANES = NB * 4;                                     // of a row
    const int part = lane % LANES, col = n0 + wn * NB * 32 + part * 8;
    float columns[8], added[8];
    if constexpr (!PARTIAL) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            columns[i] = args.finish.of_column(min(col + i, N - 1));
            added[i] = args.finish.added(min(col + i, N - 1));
        }
    }
    T* const d = PARTIAL ? reinterpret_cast<T*>(args.parts) + (int64_t)split * M * N : static_cast<T*>(args.d);
    const int64_t ldd = PARTIAL ? N : args.ldd;
    const bool aligned = ((reinterpret_cast<uintptr_t>(d) | (uintptr_t)(ldd * (int64_t)sizeof(T))) & 15) == 0;
#pragma unroll
    for (int m = 0; m < MB; ++m) {
#pragma unroll
        for (int n = 0; n < NB; ++n)
#pragma unroll
            for (int q = 0; q < 4; ++q)
                *reinterpret_cast<i32x4*>(own + (lane & 31) * ROW + (n * 32 + 8 * q + 4 * (lane >> 5)) * 4) =
                    i32x4{acc[n][m][4 * q], acc[n][m][4 * q + 1], acc[n][m][4 * q + 2], acc[n][m][4 * q + 3]};
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
#pragma unroll
        for (int i = 0; i < 32 * LANES / 64; ++i) {
            const int r = i * (64 / LANES) + lane / LANES, row = m0 + (wm * MB + m) * 32 + r;
            if (row >= M) continue;
            const i32x4 lo = *reinterpret_cast<const i32x4*>(own + r * ROW + part * 32), hi = *reinterpret_cast<const i32x4*>(own + r * ROW + part * 32 + 16);
            T* const at = d + (int64_t)row * ldd + col;
            if constexpr (PARTIAL) {
                if (aligned && col + 8 <= N) {
                    *reinterpret_cast<i32x4*>(at) = lo;
                    *reinterpret_cast<i32x4*>(at + 4) = hi;
                } else {
#pragma unroll
                    for (int e = 0; e < 8; ++e)
                        if (col + e < N) at[e] = e < 4 ? lo[e & 3] : hi[e & 3];
                }
            } else {
                const float of_row = args.finish.of_row(row);
                float v[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) v[e] = Finish::value(e < 4 ? lo[e & 3] : hi[e & 3], of_row, columns[e], added[e]);
                store8(at, v, N - col, aligned);
            }
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
    }
}

}  // namespace i8
}  // namespace anr
