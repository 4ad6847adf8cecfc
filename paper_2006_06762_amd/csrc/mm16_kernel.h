// Matrix products of 16-bit types on the matrix pipes, D[m][n] = sum_k X[m][k] W[n][k], for the products of the gated
// feed-forward block: sums in float32, one rounding where they are stored.  What the next product takes (h; dg, du and h) is rounded to the element type
// there: the matrix pipes take 16 bits, and as two numbers of 16 bits each it would be twice that product and twice the traffic between them.  The result of a
// block is then off by 1.4 times the rounding that it would have with float32 in between (0.0023 for 0.0017 of it in bf16).
//
// Each operand lies in memory with k contiguous (K_ROWS: rows of k) or with its own index contiguous (K_COLUMNS: rows
// are k).  A work-group takes a tile of BM x BN, its waves WM x WN parts of it in blocks of 32 x 32
// (v_mfma_f32_32x32x16), and walks k in chunks of 64: global -> registers -> LDS -> operands, with two LDS buffers, so that
// one is multiplied while the other is filled and the loads of the chunk after that are on their way.
//
// LDS.  K_ROWS: 128 bytes of k per row, 16-byte units exchanged by pairs of rows (unit ^ row / 2 % 8): two rows fill the 64
// banks, and sixteen rows' same unit, which an operand read takes together, lie in different ones (exchanged by row % 8, rows
// eight apart met in theirs: gate and up of 4096 x 1024 -> 2816 with tiles of 128 in 61 us, so 58; with tiles of 256, which
// wait for the matrix pipes, no difference).  K_COLUMNS: rows of k as they come, 64 bytes apart from the next one beyond
// their length; ds_read_b64_tr_b16 turns 4 k x 16 columns as it reads, each lane gets four k of its column, and the four
// rows of such a read are in different banks.
//
// W is the instruction's first operand: register r of a lane is then n = 8 (r / 4) + 4 (lane / 32) + r % 4 of the block and
// m = lane % 32: four neighbouring columns of a row of D.
#pragma once
#include "anr_kernels.h"
#include "element_types.h"

namespace anr {
namespace mm16 {

typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef half_t f16x8 __attribute__((ext_vector_type(8)));
typedef bf16_t b16x8 __attribute__((ext_vector_type(8)));

constexpr int BK = 64;                          // k of a chunk
constexpr uint32_t kNowhere = 0x80000000u;      // byte offset past every descriptor's extent: loads zeros
constexpr int kExtent = 0x7fffffff;

__device__ __forceinline__ f32x16 mfma(u32x4 a, u32x4 b, f32x16 c, half_t)
{
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
}
__device__ __forceinline__ f32x16 mfma(u32x4 a, u32x4 b, f32x16 c, bf16_t)
{
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(b16x8, a), __builtin_bit_cast(b16x8, b), c, 0, 0, 0);
}

enum Kind { K_ROWS, K_COLUMNS };
enum Epilogue {
    STORE,          // D in the element type
    PARTIAL,        // D in float32, [split][M][N] packed
    GATED,          // W's rows alternate by 32 between two matrices: act(D of the first) * D of the second
    GATED_BACKWARD  // D is dh: gradients of gate and up, and h
};

// ALIGNED kernels read 16-byte units: pointers and leading dimensions are whole units, and where an extent is none, its rows go on in zeros
// to the end of their last unit (zeros matter for k only).
//
// One product.  Two pointers of an operand: K_ROWS of GATED: gate's and up's weights; else the sum runs over
// `segments` pairs of operands of K each.
struct Problem {
    const void* x[2];
    const void* w[2];
    void* d;
    int64_t ldx, ldw, ldd;
    int M, N, K;
    int segments;
    int tiles_m, tiles_n;
};

struct Args {
    Problem p[3];
    int problems;
    int first_tile[4];              // of each problem, and of the one behind the last
    int band;                       // tiles are walked in bands of so many rows of tiles
    int splits;                     // work-groups that share a tile's k (PARTIAL)
    int act;
    // GATED: where gate and up go (or null); GATED_BACKWARD: gate and up, and where dg, du and h go (leading dimensions
    // ld_pre and problem 0's ldd)
    void *gate, *up;
    int64_t ld_pre;
    void *du, *h;
    int64_t ld_h;
    // of D, du and h in the workspace (GATED, GATED_BACKWARD): their last unit is written whole, zeros behind N
    bool whole_rows;
};

// An operand of R rows (its own index) in LDS.
template <Kind KIND, int R>
struct Image {
    static constexpr int ROW = KIND == K_ROWS ? BK * 2 : R * 2 + 64;
    static constexpr int BYTES = (KIND == K_ROWS ? R : BK) * ROW;
};

template <int BM, int BN, Kind XK, Kind WK>
constexpr size_t lds_bytes() { return 2 * (size_t)(Image<XK, BM>::BYTES + Image<WK, BN>::BYTES); }

// The units of a chunk in three parts.
constexpr int part_of(int units, int part) { return (units * part + 2) / 3; }

// Global -> registers -> LDS of one operand's chunk by NT threads.
template <typename T, Kind KIND, int R, int NT, bool ALIGNED, bool PAIRED>
struct Stager {
    static constexpr int UNITS = R * BK / 8 / NT;                     // 16-byte units of a thread
    static constexpr int ROW_UNITS = KIND == K_ROWS ? BK / 8 : R / 8; // units of a row of memory
    static_assert(R * BK / 8 % NT == 0 && NT % ROW_UNITS == 0, "whole units for every thread");
    const char* base;               // of the tile: element (first row, k = 0)
    int64_t other;                  // bytes from there to the second matrix
    int64_t ld;                     // elements
    int own, K;                     // rows (own index) from the tile's first on; k
    int first;                      // this thread's row of memory in the first unit, and its unit in the row
    int unit;
    uint32_t offset[UNITS];         // bytes from the chunk's base, or nowhere
    int which;                      // PAIRED: the matrix of unit 0 (units of a thread alternate by NT / 8 rows)
    u32x4 data[UNITS];

    // `rows`: extent of the operand's own index; `row0`: the tile's first
    __device__ __forceinline__ void init(const void* p0, const void* p1, int64_t ld_, int row0, int rows, int k, int tid)
    {
        ld = ld_;
        own = rows - row0;
        K = k;
        first = tid / ROW_UNITS;
        unit = tid % ROW_UNITS;
        const int64_t start = KIND == K_ROWS ? (int64_t)row0 * ld : row0;
        base = static_cast<const char*>(p0) + 2 * start;
        other = static_cast<const char*>(p1) - static_cast<const char*>(p0);
        if (KIND == K_ROWS) {
#pragma unroll
            for (int i = 0; i < UNITS; ++i) {
                int r = first + i * (NT / ROW_UNITS);
                if (PAIRED) r = (r >> 6) * 32 + (r & 31);
                offset[i] = (uint32_t)(min(r, own - 1) * ld * 2) + unit * 16;
            }
            which = PAIRED ? __builtin_amdgcn_readfirstlane((first >> 5) & 1) : 0;
        } else {
            const int column = ALIGNED ? min(unit * 8, ((own + 7) & ~7) - 8) : unit * 8;
#pragma unroll
            for (int i = 0; i < UNITS; ++i) offset[i] = (uint32_t)((first + i * (NT / ROW_UNITS)) * ld * 2) + column * 2;
            which = 0;
        }
    }
    __device__ __forceinline__ int matrix_of(int i) const { return PAIRED ? (which + i * (NT / ROW_UNITS) / 32) & 1 : 0; }

    // units FIRST to LAST - 1 of the chunk of k from k0 on, of segment `seg`
    template <int FIRST, int LAST>
    __device__ __forceinline__ void load(int k0, int seg)
    {
#pragma unroll
        for (int i = FIRST; i < LAST; ++i) {
            const char* const b = base + ((PAIRED ? matrix_of(i) : seg) ? other : 0) + 2 * (KIND == K_ROWS ? (int64_t)k0 : k0 * ld);
            const __amdgpu_buffer_rsrc_t rsrc = __builtin_amdgcn_make_buffer_rsrc(const_cast<char*>(b), 0, kExtent, 0x00020000);
            const int k = KIND == K_ROWS ? k0 + unit * 8 : k0 + first + i * (NT / ROW_UNITS);
            if (ALIGNED) {
                data[i] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(rsrc, (int)(k < K ? offset[i] : kNowhere), 0, 0));
            } else {
                uint16_t e[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const bool in = KIND == K_ROWS ? k + j < K : k < K && unit * 8 + j < own;
                    e[j] = __builtin_amdgcn_raw_buffer_load_b16(rsrc, (int)(in ? offset[i] + 2 * j : kNowhere), 0, 0);
                }
#pragma unroll
                for (int j = 0; j < 4; ++j) data[i][j] = e[2 * j] | (uint32_t)e[2 * j + 1] << 16;
            }
        }
    }
    template <int FIRST, int LAST>
    __device__ __forceinline__ void store(char* lds) const
    {
#pragma unroll
        for (int i = FIRST; i < LAST; ++i) {
            const int r = first + i * (NT / ROW_UNITS);
            const int at = KIND == K_ROWS ? r * Image<KIND, R>::ROW + ((unit ^ ((r >> 1) & 7)) * 16) : r * Image<KIND, R>::ROW + unit * 16;
            *reinterpret_cast<u32x4*>(lds + at) = data[i];
        }
    }
};

// Eight k from 16 step + 8 (lane / 32) on of row `row0 + lane % 32`.
template <Kind KIND, int R>
__device__ __forceinline__ u32x4 operand(const char* lds, int row0, int step, int lane)
{
    if (KIND == K_ROWS) {
        const int r = row0 + (lane & 31), u = 2 * step + (lane >> 5);
        return *reinterpret_cast<const u32x4*>(lds + r * Image<KIND, R>::ROW + ((u ^ ((r >> 1) & 7)) * 16));
    }
    typedef __attribute__((address_space(3))) s16x4 lds_t;
    const int j = lane & 15;
    const char* const at = lds + (step * 16 + (lane >> 5) * 8 + (j >> 2)) * Image<KIND, R>::ROW + (row0 + ((lane >> 4) & 1) * 16 + (j & 3) * 4) * 2;
    const u32x2 lo = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_t*)(uintptr_t)at));
    const u32x2 hi = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_t*)(uintptr_t)(at + 4 * Image<KIND, R>::ROW)));
    return u32x4{lo[0], lo[1], hi[0], hi[1]};
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
template <typename T>
__device__ __forceinline__ void load8(const T* p, float (&v)[8], int in, bool aligned)
{
    if (aligned && in >= 8) {
        load_floats<T, 8>(p, v);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = i < in ? to_float(p[i]) : 0.f;
    }
}

// store8 to the workspace: with whole_rows the last unit of a row whole, with zeros.
template <typename T>
__device__ __forceinline__ void store_workspace(T* p, float (&v)[8], int in, bool aligned, bool whole_rows)
{
    if (whole_rows && in > 0 && in < 8) {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = i < in ? v[i] : 0.f;
        in = 8;
    }
    store8(p, v, in, aligned);
}

// G groups of waves take a tile's chunks in turn, each with buffers and sums of its own, and join the sums in LDS: for products with
// about as many tiles as CUs, whose work-groups are alone on theirs.
template <typename T, int BM, int BN, int WM, int WN, int G, Kind XK, Kind WK, Epilogue EPI, bool ALIGNED>
__global__ __launch_bounds__(64 * WM * WN * G, 64 * WM * WN * G / 256) void product_kernel(const Args args)
{
    constexpr int NT = 64 * WM * WN, MB = BM / (32 * WM), NB = BN / (32 * WN);
    constexpr int XBYTES = Image<XK, BM>::BYTES, BUF = XBYTES + Image<WK, BN>::BYTES;
    constexpr bool PAIRED = EPI == GATED;
    constexpr int TILE_N = PAIRED ? BN / 2 : BN;                      // columns of D in a tile
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
    const int split = EPI == PARTIAL ? id % args.splits : 0;
    if (EPI == PARTIAL) id /= args.splits;
    const int which = (args.problems > 1 && id >= args.first_tile[1]) + (args.problems > 2 && id >= args.first_tile[2]);
    const Problem& p = args.p[which];
    id -= args.first_tile[which];
    const int band = id / (args.band * p.tiles_n), rows = min(args.band, p.tiles_m - band * args.band), in_band = id - band * args.band * p.tiles_n;
    const int m0 = (band * args.band + in_band % rows) * BM, n0 = (in_band / rows) * TILE_N;
    const int M = p.M, N = p.N, K = p.K;

    Stager<T, XK, BM, NT, ALIGNED, false> sx;
    Stager<T, WK, BN, NT, ALIGNED, PAIRED> sw;
    sx.init(p.x[0], p.x[1], p.ldx, m0, M, K, tid);
    sw.init(p.w[0], p.w[1], p.ldw, n0, N, K, tid);

    const int chunks = (K + BK - 1) / BK, all = chunks * (PAIRED ? 1 : p.segments);
    int c0 = 0, c1 = all;
    if (EPI == PARTIAL) {
        c0 = (int)((int64_t)all * split / args.splits);
        c1 = (int)((int64_t)all * (split + 1) / args.splits);
    }
    // Chunks past the last one load zeros or what is not used: no branch in the loop
    using SX = decltype(sx);
    using SW = decltype(sw);
    auto load = [&](int c, auto part) {
        constexpr int P = decltype(part)::value;
        const int seg = !PAIRED && c >= chunks;
        const int k0 = G > 1 && c >= c1 ? K : (c - (seg ? chunks : 0)) * BK;
        sx.template load<part_of(SX::UNITS, P), part_of(SX::UNITS, P + 1)>(k0, seg);
        sw.template load<part_of(SW::UNITS, P), part_of(SW::UNITS, P + 1)>(k0, seg);
    };
    auto store = [&](int buf, auto part) {
        constexpr int P = decltype(part)::value;
        sx.template store<part_of(SX::UNITS, P), part_of(SX::UNITS, P + 1)>(lds + buf * BUF);
        sw.template store<part_of(SW::UNITS, P), part_of(SW::UNITS, P + 1)>(lds + buf * BUF + XBYTES);
    };
    using P0 = std::integral_constant<int, 0>;
    using P1 = std::integral_constant<int, 1>;
    using P2 = std::integral_constant<int, 2>;

    f32x16 acc[NB][MB];
#pragma unroll
    for (int n = 0; n < NB; ++n)
#pragma unroll
        for (int m = 0; m < MB; ++m)
#pragma unroll
            for (int r = 0; r < 16; ++r) acc[n][m][r] = 0.f;

    // A chunk has four steps of 16 k.  The operands of a step are read from LDS while the one before it is multiplied; the next
    // chunk's units go to the other buffer in the first three steps, each followed by the load of the unit of the chunk after that, and
    // the barrier comes before the fourth, in which the first operands of the next chunk are read.
    u32x4 xv[2][MB], wv[2][NB];
    auto operands = [&](int set, int buf, int s) {
        const char* const x = lds + buf * BUF;
#pragma unroll
        for (int n = 0; n < NB; ++n) wv[set][n] = operand<WK, BN>(x + XBYTES, (wn * NB + n) * 32, s, lane);
#pragma unroll
        for (int m = 0; m < MB; ++m) xv[set][m] = operand<XK, BM>(x, (wm * MB + m) * 32, s, lane);
    };
    auto multiply = [&](int set) {
#pragma unroll
        for (int n = 0; n < NB; ++n)
#pragma unroll
            for (int m = 0; m < MB; ++m) acc[n][m] = mfma(wv[set][n], xv[set][m], acc[n][m], T{});
    };
    // what goes between the matrix instructions of a step: `reads` operands, then `units` stores and loads
    constexpr int kReads = (XK == K_ROWS ? MB : 2 * MB) + (WK == K_ROWS ? NB : 2 * NB);
    auto interleave = [&](auto units_c) {
        constexpr int units = decltype(units_c)::value, all_ops = kReads + 2 * units, N_ = MB * NB;
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
    if (c0 < c1) {
        const int first = c0 + group, rounds = (c1 - c0 + G - 1) / G;
        load(first, P0{});
        load(first, P1{});
        load(first, P2{});
        store(0, P0{});
        store(0, P1{});
        store(0, P2{});
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
                store(buf ^ 1, part);
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
    }
    __syncthreads();
    if constexpr (G > 1) {
        static_assert(G == 2 && (size_t)BM * BN * 4 <= 2 * G * (size_t)BUF, "the sums of one group fit the chunks' room");
        f32x16* const other = reinterpret_cast<f32x16*>(shared) + (wave * NB * MB) * 64 + lane;
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

    // The sums leave through LDS, 32 rows of a wave at a time, so that eight lanes read and write 128 bytes of a row
    // (GATED: four lanes 64 bytes).  From the registers it would be 8 bytes a row: dh with its three results and two operands
    // took 1.27 ms at 8192 x 11264 x 4096, of which 0.56 behind the products.
    constexpr int ROW = NB * 128 + 16;                                // bytes; the 16 put eight rows' same column in different banks
    static_assert((size_t)(NT / 64) * 32 * ROW <= lds_bytes<BM, BN, XK, WK>(), "fits the chunks' room");
    char* const own = lds + wave * 32 * ROW;
    constexpr int LANES = (PAIRED ? NB / 2 : NB) * 4;                 // of a row
    const int part = lane % LANES;
    auto emit = [&](auto f) {
#pragma unroll
        for (int m = 0; m < MB; ++m) {
#pragma unroll
            for (int n = 0; n < NB; ++n)
#pragma unroll
                for (int q = 0; q < 4; ++q)
                    *reinterpret_cast<f32x4*>(own + (lane & 31) * ROW + (n * 32 + 8 * q + 4 * (lane >> 5)) * 4) =
                        f32x4{acc[n][m][4 * q], acc[n][m][4 * q + 1], acc[n][m][4 * q + 2], acc[n][m][4 * q + 3]};
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            __builtin_amdgcn_wave_barrier();
#pragma unroll
            for (int i = 0; i < 32 * LANES / 64; ++i) {
                const int r = i * (64 / LANES) + lane / LANES, row = m0 + (wm * MB + m) * 32 + r;
                if (row < M) f(row, own + r * ROW);
            }
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            __builtin_amdgcn_wave_barrier();
        }
    };
    auto eight = [&](const char* at, float (&v)[8]) {
        const f32x4 lo = *reinterpret_cast<const f32x4*>(at), hi = *reinterpret_cast<const f32x4*>(at + 16);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            v[i] = lo[i];
            v[4 + i] = hi[i];
        }
    };
    auto whole = [](const void* q, int64_t ld) { return ((reinterpret_cast<uintptr_t>(q) | (uintptr_t)(2 * ld)) & 15) == 0; };
    if constexpr (EPI == STORE) {
        T* const d = static_cast<T*>(p.d);
        const bool aligned = whole(d, p.ldd);
        const int col = n0 + wn * NB * 32 + part * 8;
        emit([&](int row, const char* at) {
            float v[8];
            eight(at + part * 32, v);
            store8(d + (int64_t)row * p.ldd + col, v, N - col, aligned);
        });
    } else if constexpr (EPI == PARTIAL) {
        float* const d = static_cast<float*>(p.d) + (int64_t)split * M * N;
        const int col = n0 + wn * NB * 32 + part * 8;
        emit([&](int row, const char* at) {
            float v[8];
            eight(at + part * 32, v);
            store8(d + (int64_t)row * N + col, v, N - col, N % 8 == 0);
        });
    } else if constexpr (EPI == GATED) {
        static_assert(NB % 2 == 0, "blocks of gate and of up");
        T* const d = static_cast<T*>(p.d);
        T *const gate = static_cast<T*>(args.gate), *const up = static_cast<T*>(args.up);
        const bool aligned = whole(d, p.ldd), aligned_pre = whole(gate, args.ld_pre) && whole(up, args.ld_pre);
        auto store_unit = [&](T* at, float (&v)[8], bool aligned) { store_workspace(at, v, N - (n0 + wn * NB * 16 + part * 8), aligned, args.whole_rows); };
        const int col = n0 + wn * NB * 16 + part * 8, in_lds = (part >> 2) * 256 + (part & 3) * 32;
        device_activation(args.act, [&](auto act) {
            emit([&](int row, const char* at) {
                float g[8], u[8], h[8];
                eight(at + in_lds, g);
                eight(at + in_lds + 128, u);
#pragma unroll
                for (int e = 0; e < 8; ++e) h[e] = activation<decltype(act)::value, true>(g[e]) * u[e];
                if (gate) {
                    store8(gate + (int64_t)row * args.ld_pre + col, g, N - col, aligned_pre);
                    store8(up + (int64_t)row * args.ld_pre + col, u, N - col, aligned_pre);
                }
                store_unit(d + (int64_t)row * p.ldd + col, h, aligned);
            });
        });
    } else {
        T* const d = static_cast<T*>(p.d);
        T *const du = static_cast<T*>(args.du), *const h = static_cast<T*>(args.h);
        const T *const gate = static_cast<const T*>(args.gate), *const up = static_cast<const T*>(args.up);
        const bool aligned = whole(d, p.ldd) && whole(du, p.ldd) && whole(h, args.ld_h), aligned_pre = whole(gate, args.ld_pre) && whole(up, args.ld_pre);
        const int col = n0 + wn * NB * 32 + part * 8;
        auto store_unit = [&](T* at, float (&v)[8], bool aligned) { store_workspace(at, v, N - col, aligned, args.whole_rows); };
        device_activation(args.act, [&](auto act) {
            emit([&](int row, const char* at) {
                float g[8], u[8], dh[8], hh[8];
                load8(gate + (int64_t)row * args.ld_pre + col, g, N - col, aligned_pre);
                load8(up + (int64_t)row * args.ld_pre + col, u, N - col, aligned_pre);
                eight(at + part * 32, dh);
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    float slope;
                    const float a = activation_and_slope<decltype(act)::value, true>(g[e], slope);
                    hh[e] = a * u[e];
                    g[e] = dh[e] * u[e] * slope;
                    u[e] = dh[e] * a;
                }
                store_unit(d + (int64_t)row * p.ldd + col, g, aligned);
                store_unit(du + (int64_t)row * p.ldd + col, u, aligned);
                store_unit(h + (int64_t)row * args.ld_h + col, hh, aligned);
            });
        });
    }
}

}  // namespace mm16
}  // namespace anr
