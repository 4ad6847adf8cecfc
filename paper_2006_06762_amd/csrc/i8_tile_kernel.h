// Products of 8-bit integers in tiles on the matrix pipes (i8_device.h).
//
// A work-group takes a tile of BM x BN, its waves WM x WN parts of it in blocks of 32 x 32 (v_mfma_i32_32x32x32_i8), and walks k in chunks of BK
// bytes, which go from memory into LDS without a register between, STAGES chunks ahead of their use in as many buffers.
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

// Bytes of LDS of a work-group: STAGES chunks of 128 k of both operands' rows, and the rows' first words where these are loose.
template <int BM, int BN, int WAVES, int STAGES, bool LOOSE>
constexpr size_t tile_bytes() { return (size_t)STAGES * (BM + BN) * 128 + (LOOSE ? 2 * WAVES * 256 : 0); }

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
    __device__ __forceinline__ i32x4& of(int set, int i) { return i < NB ? wv[set][i] : xv[set][i - NB]; }
    // only the first `in` k of a step's 32 count
    __device__ __forceinline__ void cut_to(int set, int in, int lane)
    {
#pragma unroll
        for (int m = 0; m < MB; ++m) cut(xv[set][m], in - (lane >> 5) * kUnit);
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

// Rows that lie in LDS from their second word on, whose first starts up to three bytes ahead of them: an operand is sixteen bytes from the last word of the unit before on. The lanes of the lower half
// have that of the upper half's unit of the step before, which is kept, those of the upper half that of the lower half's.
template <int OPERANDS>
struct Shift {
    int before[OPERANDS];
    uint32_t bytes[OPERANDS];
    __device__ __forceinline__ void put_right(i32x4& v, int i, int lane)
    {
        const auto swapped = __builtin_amdgcn_permlane32_swap((uint32_t)before[i], (uint32_t)v[3], false, false);
        const int word = (int)(lane < 32 ? swapped[1] : swapped[0]);
        before[i] = v[3];
        v = behind_byte(v, word, bytes[i]);
    }
};

// What goes between the matrix instructions of a step: `READS` reads of operands, as early as one a matrix instruction where there are enough.
template <int MULTIPLIES, int READS>
__device__ __forceinline__ void interleave()
{
    int done = 0;
#pragma unroll
    for (int i = 0; i < MULTIPLIES; ++i) {
        __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
#pragma unroll
        for (; done < READS && done < (READS < MULTIPLIES ? i + 1 : (i + 1) * READS / MULTIPLIES); ++done) __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
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

// Rows R of one operand as the WAVES waves of a group load them to LDS: a load is 1 KB, whole rows of BK bytes.  They start at whole words; LOOSE: anywhere, and are loaded from the second word that
// has any of theirs on, the first ones once, R / WAVES a wave.
template <int R, int WAVES, int BK, bool LOOSE>
struct Feed {
    static constexpr int PER_ROW = BK / kUnit, ROWS = 64 / PER_ROW, LOADS = R / ROWS / WAVES, STARTS = R / WAVES;
    static_assert(R % (ROWS * WAVES) == 0 && STARTS <= 64, "whole loads for every wave");
    i32x4 descriptor;
    int extent, wave, last;
    uint32_t ahead, pitch, offset[LOADS];        // ahead: bytes of a word in front of the first row
    // The extent ends with the rows that exist: words past it are zeros.
    __device__ __forceinline__ void init(const int8_t* p, int64_t ld, int row0, int rows, int K, int wave_, int lane)
    {
        const int8_t* const base = p + row0 * ld;
        last = min(R, rows - row0) - 1;
        ahead = LOOSE ? (uint32_t)reinterpret_cast<uintptr_t>(base) & 3 : 0;
        pitch = (uint32_t)ld;
        descriptor = descriptor_of(base - ahead);
        extent = settled(__builtin_amdgcn_readfirstlane(((int)ahead + last * (int)ld + K + 3) & ~3));
        wave = wave_;
#pragma unroll
        for (int i = 0; i < LOADS; ++i) {
            const int r = (i * WAVES + wave) * ROWS + lane / PER_ROW;
            offset[i] = (LOOSE ? (start_of(r) & ~3u) + 4 : start_of(r)) + place_of<BK>(r, lane % PER_ROW) * kUnit;
        }
    }
    __device__ __forceinline__ uint32_t start_of(int row) const { return ahead + (uint32_t)min(row, last) * pitch; }
    __device__ __forceinline__ void limit(bool any) { descriptor[2] = any ? extent : 0; }
    __device__ __forceinline__ void load(int i, int k0, uint32_t lds) const { load_to_lds(descriptor, offset[i], k0, lds + (i * WAVES + wave) * 1024); }
    __device__ __forceinline__ void load_starts(int k0, uint32_t lds, int lane) const
    {
        load_word_to_lds(descriptor, start_of(wave * STARTS + min(lane, STARTS - 1)) & ~3u, k0, lds + wave * 256);
    }
    static __device__ __forceinline__ int word_of(int row) { return row / STARTS * 256 + row % STARTS * 4; }
};

// T: D's type; int for sums that go to `parts`.  Memory to LDS without a register between.  A buffer is loaded again as soon as all waves have read it, for the chunk STAGES further on.
//
// LOOSE: rows start at any byte.  They are loaded by whole words and put right when they are operands (Shift), by seven instructions of the vector units each
// (through registers, by 16-byte loads at any address, which issue a lane a clock, 768 x 515 -> 1408 8.5 us, so 6.6; 768 x 8193 -> 1408 39.8, 34.8; 8192 x 8193 -> 4096 284, 285; with the word behind a unit read
// from LDS beside it 331).
template <typename T, int BM, int BN, int WM, int WN, int BK, int STAGES, bool LOOSE>
__global__ __launch_bounds__(64 * WM * WN, 64 * WM * WN / 256) void tile_kernel(const Args args)
{
    constexpr bool PARTIAL = std::is_same_v<T, int>;
    constexpr int WAVES = WM * WN, MB = BM / (32 * WM), NB = BN / (32 * WN), STEPS = BK / 32;
    constexpr int XBYTES = BM * BK, BUF = XBYTES + BN * BK, STARTS = STAGES * BUF;
    extern __shared__ __attribute__((aligned(1024))) char lds[];
    const uint32_t lds_at = settled(__builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)lds));
    const int tid = threadIdx.x, lane = tid & 63, wave = settled(__builtin_amdgcn_readfirstlane(tid >> 6)), wm = wave / WN, wn = wave % WN;
    const int K = args.K, chunks = (K + BK - 1) / BK;
    const Place at(args, BM, BN, chunks, PARTIAL);

    Feed<BM, WAVES, BK, LOOSE> fx;
    Feed<BN, WAVES, BK, LOOSE> fw;
    fx.init(args.x, args.ldx, at.m0, args.M, K, wave, lane);
    fw.init(args.w, args.ldw, at.n0, args.N, K, wave, lane);
    constexpr int XLOADS = decltype(fx)::LOADS, LOADS = XLOADS + decltype(fw)::LOADS;
    auto load = [&](int i, int c, int buf) {
        if (i < XLOADS) fx.load(i, c * BK, lds_at + buf * BUF);
        else fw.load(i - XLOADS, c * BK, lds_at + buf * BUF + XBYTES);
    };

    Wave<MB, NB> w;
    w.clear();
    const char* const x_rows = lds + wm * MB * 32 * BK;
    const char* const w_rows = lds + XBYTES + wn * NB * 32 * BK;
    Shift<MB + NB> shift;
    auto read = [&](int set, int buf, int s, int i) { w.template read<BK>(set, x_rows + buf * BUF, w_rows + buf * BUF, s, lane, i); };
    auto read_all = [&](int set, int buf, int s) {
#pragma unroll
        for (int i = 0; i < NB + MB; ++i) read(set, buf, s, i);
    };
    auto put_right = [&](int set) {
        if (!LOOSE) return;
#pragma unroll
        for (int i = 0; i < NB + MB; ++i) shift.put_right(w.of(set, i), i, lane);
    };

    // Loads of chunks past the last one are of descriptors without an extent, which read nothing: no branch in the loop, and as many loads on their way in its last
    // rounds as in the others.
    const int rounds = at.c1 - at.c0, first = settled(at.c0);
    // The loads of a chunk start in the step behind the barrier that frees its buffer; half of them go into the step after that (4096 x 4096 x 4096 by four waves: all in
    // the first one 73 us, so 67.5; a third or two thirds level).
    constexpr int LATER = LOADS / 2, MANY = MB * NB > MB + NB ? MB * NB : MB + NB;
    // Loose operands are put right in the step that reads them where that has matrix instructions enough (8192 x 8193 -> 4096 291 us, so 285; parts of one block 34.6, so 38).
    constexpr bool AHEAD = LOOSE && MB * NB >= 8;
    if (LOOSE) {
        fx.limit(true);
        fw.limit(true);
        fx.load_starts(first * BK, lds_at + STARTS, lane);
        fw.load_starts(first * BK, lds_at + STARTS + WAVES * 256, lane);
    }
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
    read_all(0, 0, 0);
    if (LOOSE) {
#pragma unroll
        for (int i = 0; i < MB + NB; ++i) {
            const int r = (i < NB ? wn * NB + i : wm * MB + i - NB) * 32 + (lane & 31);
            shift.before[i] = *reinterpret_cast<const int*>(lds + STARTS + (i < NB ? WAVES * 256 + decltype(fw)::word_of(r) : decltype(fx)::word_of(r)));
            shift.bytes[i] = i < NB ? fw.start_of(r) : fx.start_of(r);
        }
        if (AHEAD) put_right(0);
    }
    int buf = 0, r = 0;
    // A step multiplies the operands of one set while those of the next step are read into the other, and COUNT loads, from number `from` on, go to buffer `to`.
    auto step = [&](int set, int read_from, int read_step, auto count, int from, int c, int to) {
        constexpr int COUNT = decltype(count)::value;
        if (!AHEAD) put_right(set);
        if constexpr (COUNT == 0 && !AHEAD) {
            read_all(set ^ 1, read_from, read_step);
            w.multiply_all(set);
            interleave<MB * NB, MB + NB>();
            __builtin_amdgcn_sched_barrier(0);
        } else {
#pragma unroll
            for (int i = 0; i < MANY; ++i) {
                if (i < MB * NB) w.multiply(set, i);
                if (!AHEAD && i < MB + NB) read(set ^ 1, read_from, read_step, i);
#pragma unroll
                for (int j = 0; j < MB + NB; ++j) {
                    if (AHEAD && j / 2 == i) read(set ^ 1, read_from, read_step, j);
                    if (AHEAD && MANY / 2 + j * (MANY - MANY / 2) / (MB + NB) == i) shift.put_right(w.of(set ^ 1, j), j, lane);
                }
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
    // The last chunk, which k may end in: what lies past it counts in neither operand if it is cleared in one.
    const int in = K - (at.c1 - 1) * BK;
#pragma unroll
    for (int s = 0; s < STEPS; ++s) {
        if (s + 1 < STEPS) read_all((s & 1) ^ 1, buf, s + 1);
        if (!AHEAD) put_right(s & 1);
        if (in < BK) w.cut_to(s & 1, in - 32 * s, lane);
        w.multiply_all(s & 1);
        if (AHEAD && s + 1 < STEPS) put_right((s & 1) ^ 1);
    }
    wait_for_loads<0>();
    finish_tile<T, WM, WN, STAGES * (size_t)BUF>(args, at, w, lds, tid);
}

}  // namespace i8
}  // namespace anr
