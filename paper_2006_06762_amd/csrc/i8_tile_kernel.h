// Products of 8-bit integers in tiles on the matrix pipes (i8_device.h).
//
// A work-group takes a tile of BM x BN, its waves WM x WN parts of it in blocks of 32 x 32 (v_mfma_i32_32x32x32_i8), and walks k in chunks of BK
// bytes.  Rows that are whole 16-byte units (tile_kernel) go from memory into LDS without a register between, STAGES chunks ahead of their use in as many
// buffers; others (loose_kernel) through registers, where what lies past their end is cleared.
//
// LDS: rows of BK bytes, 16-byte units exchanged by as many rows as fill the 64 banks (unit ^ row / 2 % 8 for 128 bytes), so that the sixteen rows' same unit that
// an operand read takes together lie in different ones.  Loads write LDS in the order of the lanes: the lanes take the units of a row in that order instead.
//
// W is the instruction's first operand: register r of a lane is then n = 8 (r / 4) + 4 (lane / 32) + r % 4 of the block and m = lane % 32: four
// neighbouring columns of a row of D.
#pragma once
#include "i8_device.h"

namespace anr {
namespace i8 {

// The units of a chunk in three parts.
constexpr int part_of(int units, int part) { return (units * part + 2) / 3; }

// Global -> registers -> LDS of R rows of one operand by NT threads.
template <int R, int NT, int BK, bool CLEAR>
struct Stager {
    static constexpr int PER_ROW = BK / kUnit, UNITS = R * PER_ROW / NT;
    static_assert(R * PER_ROW % NT == 0 && NT % PER_ROW == 0, "whole units for every thread");
    const int8_t* base;             // of the tile's first row
    int K, first, unit;             // this thread's row in the first unit, its unit in the row
    uint32_t offset[UNITS];         // bytes of a row's start from the base
    u32x4 data[UNITS];

    __device__ __forceinline__ void init(const int8_t* p, int64_t ld, int row0, int rows, int k, int tid)
    {
        base = p + row0 * ld;
        K = k;
        first = tid / PER_ROW;
        unit = tid % PER_ROW;
#pragma unroll
        for (int i = 0; i < UNITS; ++i) offset[i] = (uint32_t)(min(first + i * (NT / PER_ROW), rows - row0 - 1) * ld);
    }
    // units FIRST to LAST - 1 of the chunk of k from k0 on
    template <int FIRST, int LAST>
    __device__ __forceinline__ void load(int k0)
    {
        const int start = loose_start(k0 + unit * kUnit, K);
#pragma unroll
        for (int i = FIRST; i < LAST; ++i) data[i] = load_loose(base + offset[i] + start);
    }
    template <int FIRST, int LAST>
    __device__ __forceinline__ void store(char* lds, int k0)
    {
        if (CLEAR && k0 + BK > K) {
#pragma unroll
            for (int i = FIRST; i < LAST; ++i) clear_counted(data[i], k0 + unit * kUnit, K);
        }
#pragma unroll
        for (int i = FIRST; i < LAST; ++i) {
            const int r = first + i * (NT / PER_ROW);
            *reinterpret_cast<u32x4*>(lds + r * BK + place_of<BK>(r, unit) * 16) = data[i];
        }
    }
};

// Sixteen k from 32 step + 16 (lane / 32) on of row `row0 + lane % 32`.
template <int BK>
__device__ __forceinline__ i32x4 operand(const char* lds, int row0, int step, int lane)
{
    const int r = row0 + (lane & 31), u = 2 * step + (lane >> 5);
    return *reinterpret_cast<const i32x4*>(lds + r * BK + place_of<BK>(r, u) * 16);
}

// Eight neighbouring elements of a row at any element's address (STREAMING: past L2, whole aligned units), of which `in` exist (3000 x 512 -> 3001 in bf16 one by one 28.7 us, so 14.7).
template <bool STREAMING, typename T, typename V>
__device__ __forceinline__ void store8(T* p, const V (&v)[8], int in)
{
    if (in >= 8) {
        if constexpr (STREAMING) {
            T w[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) w[i] = (T)v[i];
#pragma unroll
            for (int i = 0; i < (int)sizeof(T) / 2; ++i) {
                u32x4 q;
                __builtin_memcpy(&q, reinterpret_cast<const char*>(w) + 16 * i, 16);
                __builtin_nontemporal_store(q, reinterpret_cast<u32x4*>(p) + i);
            }
            return;
        }
        struct __attribute__((packed, aligned(sizeof(T)))) Loose { T v[8]; };
        Loose l;
#pragma unroll
        for (int i = 0; i < 8; ++i) l.v[i] = (T)v[i];
        *reinterpret_cast<Loose*>(p) = l;
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < in) p[i] = (T)v[i];
    }
}

// A work-group's tile, and the chunks of k that it takes.
struct Place {
    int m0, n0, split, c0, c1;
    __device__ __forceinline__ Place(const Args& a, int BM, int BN, int chunks, bool partial)
    {
        // Work-group ids are dealt round-robin over the 8 XCDs, each with its own L2: every XCD gets a contiguous run of tiles,
        // walked in bands of `band` rows of tiles, column by column
        const int all = (int)gridDim.x, per = all >> 3, rest = all & 7, xcd = blockIdx.x & 7, slot = blockIdx.x >> 3;
        int id = xcd * per + (xcd < rest ? xcd : rest) + slot;
        split = partial ? id % a.splits : 0;
        if (partial) id /= a.splits;
        const int band = id / (a.band * a.tiles_n), rows = min(a.band, a.tiles_m - band * a.band), in_band = id - band * a.band * a.tiles_n;
        m0 = __builtin_amdgcn_readfirstlane((band * a.band + in_band % rows) * BM);
        n0 = __builtin_amdgcn_readfirstlane((in_band / rows) * BN);
        split = __builtin_amdgcn_readfirstlane(split);
        c0 = partial ? __builtin_amdgcn_readfirstlane(chunks * split / a.splits) : 0;                    // (k has at most 1024 chunks, shared by 16 at most)
        c1 = partial ? __builtin_amdgcn_readfirstlane(chunks * (split + 1) / a.splits) : chunks;
    }
};

// A wave's part of a tile: its sums, and the operands of two steps of 32 k.
template <int MB, int NB>
struct Wave {
    i32x16 acc[NB][MB];
    i32x4 xv[2][MB], wv[2][NB];
    __device__ __forceinline__ void clear()
    {
#pragma unroll
        for (int n = 0; n < NB; ++n)
#pragma unroll
            for (int m = 0; m < MB; ++m)
#pragma unroll
                for (int r = 0; r < 16; ++r) acc[n][m][r] = 0;
    }
    // operand i of a step, of NB + MB, from the wave's rows of X and W in LDS
    template <int BK>
    __device__ __forceinline__ void read(int set, const char* x, const char* w, int step, int lane, int i)
    {
        if (i < NB) wv[set][i] = operand<BK>(w, i * 32, step, lane);
        else xv[set][i - NB] = operand<BK>(x, (i - NB) * 32, step, lane);
    }
    template <int BK>
    __device__ __forceinline__ void read_all(int set, const char* x, const char* w, int step, int lane)
    {
#pragma unroll
        for (int i = 0; i < NB + MB; ++i) read<BK>(set, x, w, step, lane, i);
    }
    __device__ __forceinline__ void multiply(int set, int i)
    {
        acc[i / MB][i % MB] = __builtin_amdgcn_mfma_i32_32x32x32_i8(wv[set][i / MB], xv[set][i % MB], acc[i / MB][i % MB], 0, 0, 0);
    }
    __device__ __forceinline__ void multiply_all(int set)
    {
#pragma unroll
        for (int i = 0; i < NB * MB; ++i) multiply(set, i);
    }
};

// What goes between the matrix instructions of a step: `READS` operands, then `UNITS` stores and loads; reads alone as early as one a matrix instruction.
template <int MULTIPLIES, int READS, int UNITS>
__device__ __forceinline__ void interleave()
{
    constexpr int all = READS + 2 * UNITS;
    int done = 0;
#pragma unroll
    for (int i = 0; i < MULTIPLIES; ++i) {
        __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
#pragma unroll
        for (; done < all && done < (UNITS == 0 && READS < MULTIPLIES ? i + 1 : (i + 1) * all / MULTIPLIES); ++done) {
            if (done < READS) __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
            else if ((done - READS) % 2 == 0) __builtin_amdgcn_sched_group_barrier(0x200, 1, 0);
            else __builtin_amdgcn_sched_group_barrier(0x020, 1, 0);
        }
    }
}

// The end of a tile: the sums leave through LDS, 32 rows of a wave at a time, so that neighbouring lanes write neighbouring units of a row.  ROOM: bytes of LDS.
template <typename T, int WM, int WN, size_t ROOM, int MB, int NB>
__device__ __forceinline__ void finish_tile(const Args& a, const Place& at, Wave<MB, NB>& w, char* lds, int tid)
{
    constexpr bool PARTIAL = std::is_same_v<T, int>;
    constexpr int NT = 64 * WM * WN;
    const int lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), wm = wave / WN, wn = wave % WN;
    const int M = a.M, N = a.N;
    auto& acc = w.acc;
    __syncthreads();
    constexpr int ROW = NB * 128 + 16;                                // bytes; the 16 put eight rows' same column in different banks
    static_assert((size_t)(NT / 64) * 32 * ROW <= ROOM, "fits the chunks' room");
    constexpr int LANES = NB * 4;                                     // of a row
    const int part = lane % LANES, col = at.n0 + wn * NB * 32 + part * 8;
    float rows[MB], columns[8], added[8];
    if constexpr (!PARTIAL) {
#pragma unroll
        for (int m = 0; m < MB; ++m) rows[m] = a.finish.of_row(min(at.m0 + (wm * MB + m) * 32 + (lane & 31), M - 1));
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            columns[i] = a.finish.of_column(min(col + i, N - 1));
            added[i] = a.finish.added(min(col + i, N - 1));
        }
    }
    T* const d = PARTIAL ? reinterpret_cast<T*>(a.parts) + (int64_t)at.split * M * N : static_cast<T*>(a.d);
    const int64_t ldd = PARTIAL ? N : a.ldd;
    by_streaming(!PARTIAL && a.streaming, [&](auto streaming) {
#pragma unroll
        for (int m = 0; m < MB; ++m) {
#pragma unroll
            for (int n = 0; n < NB; ++n)
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    char* const to = lds + wave * 32 * ROW + (lane & 31) * ROW + (n * 32 + 8 * q + 4 * (lane >> 5)) * 4;
                    if constexpr (PARTIAL) {
                        *reinterpret_cast<i32x4*>(to) = i32x4{acc[n][m][4 * q], acc[n][m][4 * q + 1], acc[n][m][4 * q + 2], acc[n][m][4 * q + 3]};
                    } else {                                          // (a row's scale is one for a lane here, those of columns are where they are read)
                        f32x4 v;
#pragma unroll
                        for (int e = 0; e < 4; ++e) v[e] = (float)acc[n][m][4 * q + e] * rows[m];
                        *reinterpret_cast<f32x4*>(to) = v;
                    }
                }
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            __builtin_amdgcn_wave_barrier();
#pragma unroll
            for (int i = 0; i < 32 * LANES / 64; ++i) {
                const int r = i * (64 / LANES) + lane / LANES, row = at.m0 + (wm * MB + m) * 32 + r;
                if (row >= M) continue;
                using Four = std::conditional_t<PARTIAL, i32x4, f32x4>;
                const char* const from = lds + wave * 32 * ROW + r * ROW + part * 32;
                const Four lo = *reinterpret_cast<const Four*>(from), hi = *reinterpret_cast<const Four*>(from + 16);
                T* const to = d + (int64_t)row * ldd + col;
                if constexpr (PARTIAL) {
                    const int v[8] = {lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
                    store8<false>(to, v, N - col);
                } else {
                    float v[8];
#pragma unroll
                    for (int e = 0; e < 8; ++e) v[e] = (e < 4 ? lo[e & 3] : hi[e & 3]) * columns[e] + added[e];
                    store8<decltype(streaming)::value>(to, v, N - col);
                }
            }
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            __builtin_amdgcn_wave_barrier();
        }
    });
}

// T: D's type; int for sums that go to `parts`.
//
// Rows at any address and of any length from 16 on: global -> registers -> LDS -> operands, with two buffers, so that one is multiplied while the other
// is filled and the loads of the chunk after that are on their way (two chunks on their way to the registers: 768 x 515 -> 1408 8.1 us, so 9.5).
template <typename T, int BM, int BN, int WM, int WN>
__global__ __launch_bounds__(64 * WM * WN, 64 * WM * WN / 256) void loose_kernel(const Args args)
{
    constexpr bool PARTIAL = std::is_same_v<T, int>;
    constexpr int BK = 128, NT = 64 * WM * WN, MB = BM / (32 * WM), NB = BN / (32 * WN);
    constexpr int XBYTES = BM * BK, BUF = XBYTES + BN * BK;
    extern __shared__ __attribute__((aligned(16))) char lds[];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int K = args.K, chunks = (K + BK - 1) / BK;
    const Place at(args, BM, BN, chunks, PARTIAL);

    Stager<BM, NT, BK, true> sx;
    Stager<BN, NT, BK, false> sw;
    sx.init(args.x, args.ldx, at.m0, args.M, K, tid);
    sw.init(args.w, args.ldw, at.n0, args.N, K, tid);

    // Chunks past the last one are loaded and cleared: no branch in the loop
    using SX = decltype(sx);
    using SW = decltype(sw);
    auto load = [&](int c, auto part) {
        constexpr int P = decltype(part)::value;
        sx.template load<part_of(SX::UNITS, P), part_of(SX::UNITS, P + 1)>(c * BK);
        sw.template load<part_of(SW::UNITS, P), part_of(SW::UNITS, P + 1)>(c * BK);
    };
    auto store = [&](int buf, int c, auto part) {
        constexpr int P = decltype(part)::value;
        sx.template store<part_of(SX::UNITS, P), part_of(SX::UNITS, P + 1)>(lds + buf * BUF, c * BK);
        sw.template store<part_of(SW::UNITS, P), part_of(SW::UNITS, P + 1)>(lds + buf * BUF + XBYTES, c * BK);
    };
    using P0 = std::integral_constant<int, 0>;
    using P1 = std::integral_constant<int, 1>;
    using P2 = std::integral_constant<int, 2>;
    // A chunk has four steps of 32 k.  The operands of a step are read from LDS while the one before it is multiplied; the next
    // chunk's units go to the other buffer in the first three steps, each followed by the load of the unit of the chunk after that, and
    // the barrier comes before the fourth, in which the first operands of the next chunk are read.
    Wave<MB, NB> w;
    w.clear();
    const char* const x_rows = lds + (wave / WN) * MB * 32 * BK;
    const char* const w_rows = lds + XBYTES + (wave % WN) * NB * 32 * BK;
    auto operands = [&](int set, int buf, int s) { w.template read_all<BK>(set, x_rows + buf * BUF, w_rows + buf * BUF, s, lane); };
    load(at.c0, P0{});
    load(at.c0, P1{});
    load(at.c0, P2{});
    store(0, at.c0, P0{});
    store(0, at.c0, P1{});
    store(0, at.c0, P2{});
    load(at.c0 + 1, P0{});
    load(at.c0 + 1, P1{});
    load(at.c0 + 1, P2{});
    __syncthreads();
    operands(0, 0, 0);
#pragma unroll 1
    for (int c = at.c0; c < at.c1; ++c) {
        const int buf = (c - at.c0) & 1;
        auto step = [&](auto part) {
            constexpr int S = decltype(part)::value;
            operands((S + 1) & 1, buf, S + 1);
            w.multiply_all(S & 1);
            store(buf ^ 1, c + 1, part);
            load(c + 2, part);
            interleave<MB * NB, MB + NB, part_of(SX::UNITS, S + 1) - part_of(SX::UNITS, S) + part_of(SW::UNITS, S + 1) - part_of(SW::UNITS, S)>();
            __builtin_amdgcn_sched_barrier(0);
        };
        step(P0{});
        step(P1{});
        step(P2{});
        __syncthreads();
        operands(0, buf ^ 1, 0);
        w.multiply_all(1);
        interleave<MB * NB, MB + NB, 0>();
        __builtin_amdgcn_sched_barrier(0);
    }
    finish_tile<T, WM, WN, 2 * (size_t)BUF>(args, at, w, lds, tid);
}

// Rows R of one operand as the WAVES waves of a group load them to LDS: a load is 1 KB, whole rows of BK bytes.
template <int R, int WAVES, int BK>
struct Feed {
    static constexpr int PER_ROW = BK / kUnit, ROWS = 64 / PER_ROW, LOADS = R / ROWS / WAVES;
    static_assert(R % (ROWS * WAVES) == 0, "whole loads for every wave");
    i32x4 descriptor;
    uint32_t offset[LOADS];
    int wave;
    __device__ __forceinline__ void init(const int8_t* p, int64_t ld, int row0, int rows, int wave_, int lane)
    {
        descriptor = descriptor_of(p + row0 * ld);
        wave = wave_;
#pragma unroll
        for (int i = 0; i < LOADS; ++i) {
            const int r = (i * WAVES + wave) * ROWS + lane / PER_ROW;
            offset[i] = (uint32_t)(min(r, rows - row0 - 1) * ld) + place_of<BK>(r, lane % PER_ROW) * kUnit;
        }
    }
    __device__ __forceinline__ void limit(bool any) { descriptor[2] = any ? kExtent : 0; }
    __device__ __forceinline__ void load(int i, int k0, uint32_t lds) const { load_to_lds(descriptor, offset[i], k0, lds + (i * WAVES + wave) * 1024); }
};

// Rows of whole 16-byte units (pointers, leading dimensions, K).  A buffer is loaded again as soon as all waves have read it, for the chunk STAGES further on.
template <typename T, int BM, int BN, int WM, int WN, int BK, int STAGES>
__global__ __launch_bounds__(64 * WM * WN, 64 * WM * WN / 256) void tile_kernel(const Args args)
{
    constexpr bool PARTIAL = std::is_same_v<T, int>;
    constexpr int WAVES = WM * WN, NT = 64 * WAVES, MB = BM / (32 * WM), NB = BN / (32 * WN), STEPS = BK / 32;
    constexpr int XBYTES = BM * BK, BUF = XBYTES + BN * BK;
    extern __shared__ __attribute__((aligned(1024))) char lds[];
    const uint32_t lds_at = settled(__builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)lds));
    const int tid = threadIdx.x, lane = tid & 63, wave = settled(__builtin_amdgcn_readfirstlane(tid >> 6));
    const int K = args.K, chunks = (K + BK - 1) / BK;
    const Place at(args, BM, BN, chunks, PARTIAL);

    Feed<BM, WAVES, BK> fx;
    Feed<BN, WAVES, BK> fw;
    fx.init(args.x, args.ldx, at.m0, args.M, wave, lane);
    fw.init(args.w, args.ldw, at.n0, args.N, wave, lane);
    constexpr int XLOADS = decltype(fx)::LOADS, LOADS = XLOADS + decltype(fw)::LOADS;
    auto load = [&](int i, int c, int buf) {
        if (i < XLOADS) fx.load(i, c * BK, lds_at + buf * BUF);
        else fw.load(i - XLOADS, c * BK, lds_at + buf * BUF + XBYTES);
    };

    Wave<MB, NB> w;
    w.clear();
    const char* const x_rows = lds + (wave / WN) * MB * 32 * BK;
    const char* const w_rows = lds + XBYTES + (wave % WN) * NB * 32 * BK;

    // The whole chunks; one that k ends in comes last.  Loads of chunks past them are of descriptors without an extent, which read nothing: no branch
    // in the loop, and as many loads on their way in its last rounds as in the others.
    const int rounds = min(K / BK, at.c1) - at.c0, first = settled(at.c0);
    if (rounds > 0) {
        // The loads of a chunk start in the step behind the barrier that frees its buffer; half of them go into the step after that (4096 x 4096 x 4096 by four waves: all in
        // the first one 73 us, so 67.5; a third or two thirds level).
        constexpr int LATER = LOADS / 2, MANY = MB * NB > MB + NB ? MB * NB : MB + NB;
#pragma unroll
        for (int s = 0; s < STAGES; ++s) {
            fx.limit(s < rounds);
            fw.limit(s < rounds);
#pragma unroll
            for (int i = 0; i < LOADS - (s + 1 == STAGES ? LATER : 0); ++i) load(i, first + s, s);
        }
        wait_for_loads<(STAGES - 1) * LOADS - LATER>();
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
        w.template read_all<BK>(0, x_rows, w_rows, 0, lane);
        int buf = 0, r = 0;
        // A step multiplies the operands of one set while those of the next step are read into the other, and COUNT loads, from number `from` on, go to buffer `to`.
        auto step = [&](int set, int read_from, int read_step, auto count, int from, int c, int to) {
            constexpr int COUNT = decltype(count)::value;
            if constexpr (COUNT == 0) {
                w.template read_all<BK>(set ^ 1, x_rows + read_from * BUF, w_rows + read_from * BUF, read_step, lane);
                w.multiply_all(set);
                interleave<MB * NB, MB + NB, 0>();
                __builtin_amdgcn_sched_barrier(0);
            } else {
#pragma unroll
                for (int i = 0; i < MANY; ++i) {
                    if (i < MB * NB) w.multiply(set, i);
                    if (i < MB + NB) w.template read<BK>(set ^ 1, x_rows + read_from * BUF, w_rows + read_from * BUF, read_step, lane, i);
#pragma unroll
                    for (int j = 0; j < COUNT; ++j)
                        if (j * MANY / COUNT == i) load(from + j, c, to);
                    __builtin_amdgcn_sched_barrier(0);
                }
            }
        };
        constexpr int LAST = (STEPS - 1) & 1;
        using None = std::integral_constant<int, 0>;
#pragma unroll 1
        for (; r + 1 < rounds; ++r) {
            step(0, buf, 1, std::integral_constant<int, LATER>{}, LOADS - LATER, first + r - 1 + STAGES, buf == 0 ? STAGES - 1 : buf - 1);
#pragma unroll
            for (int s = 1; s + 1 < STEPS; ++s) step(s & 1, buf, s + 1, None{}, 0, 0, 0);
            wait_for_loads<(STAGES - 2) * LOADS>();
            __builtin_amdgcn_s_barrier();
            asm volatile("" ::: "memory");
            const int next = buf + 1 == STAGES ? 0 : buf + 1;
            fx.limit(r + STAGES < rounds);
            fw.limit(r + STAGES < rounds);
            step(LAST, next, 0, std::integral_constant<int, LOADS - LATER>{}, 0, first + r + STAGES, buf);
            buf = next;
        }
#pragma unroll
        for (int s = 0; s + 1 < STEPS; ++s) step(s & 1, buf, s + 1, None{}, 0, 0, 0);
        w.multiply_all(LAST);
        wait_for_loads<0>();
    }
    if (K % BK != 0 && at.c1 == chunks) {                             // the chunk that k ends in, through registers
        __syncthreads();
        {
            Stager<BM, NT, BK, true> sx;
            Stager<BN, NT, BK, false> sw;
            sx.init(args.x, args.ldx, at.m0, args.M, K, tid);
            sw.init(args.w, args.ldw, at.n0, args.N, K, tid);
            const int k0 = (chunks - 1) * BK;
            sx.template load<0, decltype(sx)::UNITS>(k0);
            sw.template load<0, decltype(sw)::UNITS>(k0);
            sx.template store<0, decltype(sx)::UNITS>(lds, k0);
            sw.template store<0, decltype(sw)::UNITS>(lds + XBYTES, k0);
        }
        __syncthreads();
#pragma unroll
        for (int s = 0; s < STEPS; ++s) {
            w.template read_all<BK>(0, x_rows, w_rows, s, lane);
            w.multiply_all(0);
        }
    }
    finish_tile<T, WM, WN, STAGES * (size_t)BUF>(args, at, w, lds, tid);
}

}  // namespace i8
}  // namespace anr
