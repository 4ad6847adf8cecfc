// Products of a few rows X [M,K], M <= 16 TB, of 8-bit integers with a large matrix W (i8_device.h), as single tokens need them.
//
// Bound: reading W once.  A work-group takes 16 rows of W, its waves share the k in chunks of 128 and join their sums in LDS; the matrix instructions
// (v_mfma_i32_16x16x64_i8) are sixteen tokens wide, which cost nothing here.
#pragma once
#include "i8_device.h"

namespace anr {
namespace i8 {

constexpr int kRowsChunk = 128;                 // k of a wave at a time: a line of a row
constexpr int most_waves(int TB) { return TB == 1 ? 16 : TB == 2 ? 8 : 4; }      // of a work-group: their buffers fit LDS

// The results of a thread: what they are multiplied with is read before the products, whose sums [wave][TB][4][64] join at the end.  At least four waves.
template <typename T, int TB>
struct Results {
    static constexpr int MOST = TB;
    float row[MOST], column[MOST], added[MOST];
    // register e of lane l: row 4 (l / 16) + e of W, token l % 16
    static __device__ __forceinline__ int token_of(int i) { return (i >> 8) * 16 + (i & 15); }
    static __device__ __forceinline__ int column_of(int i, int n0) { return n0 + 4 * ((i >> 4) & 3) + ((i >> 6) & 3); }
    __device__ __forceinline__ void init(const Args& a, int n0)
    {
#pragma unroll
        for (int j = 0; j < MOST; ++j) {
            const int i = threadIdx.x + j * (int)blockDim.x;
            row[j] = a.finish.of_row(min(token_of(i), a.M - 1));
            column[j] = a.finish.of_column(min(column_of(i, n0), a.N - 1));
            added[j] = a.finish.added(min(column_of(i, n0), a.N - 1));
        }
    }
    __device__ __forceinline__ void store(const Args& a, const int* sums, int n0) const
    {
        const int waves = blockDim.x >> 6;
#pragma unroll
        for (int j = 0; j < MOST; ++j) {
            const int i = threadIdx.x + j * (int)blockDim.x, token = token_of(i), n = column_of(i, n0);
            if (i >= TB * 256 || token >= a.M || n >= a.N) continue;
            int v = 0;
            for (int w = 0; w < waves; ++w) v += sums[w * TB * 256 + i];
            static_cast<T*>(a.d)[token * a.ldd + n] = from_float<T>(Finish::value(v, row[j], column[j], added[j]));
        }
    }
};

// Rows go through LDS: a lane's operand is of one of sixteen rows, and loads whose neighbouring lanes are in different lines take four times as
// long to issue (32 tokens 4096 -> 11264 19.4 us straight from memory, so 13.6; 1 token 5632 -> 2048 5.4, 4.0).  Each wave has STAGES buffers of its own, of its 16 rows of W and the 16 TB rows of X, and waits for no other one but at the end.
// WHOLE: rows of whole 16-byte units (pointers, leading dimensions, K), which go from memory to LDS; others, of any length from 16 on, go through registers, a chunk ahead.
template <typename T, int TB, int STAGES, bool WHOLE>
__global__ __launch_bounds__(64 * most_waves(TB)) void stream_kernel(const Args a)
{
    constexpr int BK = kRowsChunk, STAGE = 16 * (1 + TB) * BK, LOADS = 2 * (1 + TB);
    extern __shared__ __attribute__((aligned(1024))) char lds[];                  // buffers, then sums [wave][TB][4][64]
    const uint32_t lds_at = settled(__builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)lds));
    const int tid = threadIdx.x, lane = tid & 63, wave = settled(__builtin_amdgcn_readfirstlane(tid >> 6)), waves = blockDim.x >> 6;
    const int n0 = blockIdx.x * 16;
    const i32x4 of_w = descriptor_of(a.w + n0 * a.ldw), of_x = descriptor_of(a.x);
    // A load is eight rows; a lane has one of these and one of its units
    uint32_t row[LOADS];
#pragma unroll
    for (int i = 0; i < LOADS; ++i) {
        const int r = (i < 2 ? i : i - 2) * 8 + (lane >> 3);
        row[i] = i < 2 ? (uint32_t)(min(r, a.N - 1 - n0) * a.ldw) : (uint32_t)(min(r, a.M - 1) * a.ldx);
    }
    const int unit0 = place_of<BK>(lane >> 3, lane & 7) * kUnit, unit1 = place_of<BK>(8 + (lane >> 3), lane & 7) * kUnit;
    const int chunks = (a.K + BK - 1) / BK;
    const uint32_t own = lds_at + wave * STAGES * STAGE;
    // (units past K: the last one instead, cleared in X where it is used; chunks past the last one read nothing)
    auto load = [&](int c, int stage) {
        i32x4 dw = of_w, dx = of_x;
        dw[2] = dx[2] = c < chunks ? kExtent : 0;
        const int k0 = min(c * BK + unit0, a.K - kUnit), k1 = min(c * BK + unit1, a.K - kUnit);
#pragma unroll
        for (int i = 0; i < LOADS; ++i) load_to_lds(i < 2 ? dw : dx, row[i] + (i & 1 ? k1 : k0), 0, own + stage * STAGE + i * 1024);
    };
    i32x4 acc[TB];
#pragma unroll
    for (int t = 0; t < TB; ++t) acc[t] = i32x4{0, 0, 0, 0};
    i32x4 v[2][1 + TB];
    auto read = [&](const char* at) {
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int j = 0; j < 1 + TB; ++j) {
                const int r = lane & 15;
                v[i][j] = *reinterpret_cast<const i32x4*>(at + (j * 16 + r) * BK + place_of<BK>(r, 4 * i + (lane >> 4)) * kUnit);
            }
    };
    auto multiply = [&]() {
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int t = 0; t < TB; ++t) acc[t] = __builtin_amdgcn_mfma_i32_16x16x64_i8(v[i][0], v[i][1 + t], acc[t], 0, 0, 0);
    };
    Results<T, TB> results;
    if constexpr (WHOLE) {
        load(wave, 0);
        results.init(a, n0);                                         // (in front of the loads that the first wait leaves on their way)
#pragma unroll
        for (int s = 1; s < STAGES; ++s) load(wave + s * waves, s);
        int stage = 0;
#pragma unroll 1
        for (int c = wave; c < chunks; c += waves) {
            wait_for_loads<(STAGES - 1) * LOADS>();
            read(lds + (wave * STAGES + stage) * STAGE);
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
            load(c + STAGES * waves, stage);
            stage = stage + 1 == STAGES ? 0 : stage + 1;
            if ((c + 1) * BK > a.K) {
#pragma unroll
                for (int i = 0; i < 2; ++i)
#pragma unroll
                    for (int t = 0; t < TB; ++t)
                        if (c * BK + (4 * i + (lane >> 4)) * kUnit >= a.K) v[i][1 + t] = i32x4{0, 0, 0, 0};
            }
            multiply();
        }
    } else {
        u32x4 data[STAGES][LOADS];
        const int8_t* const w0 = a.w + n0 * a.ldw;
        auto load_loosely = [&](u32x4 (&to)[LOADS], int c) {
            const int start0 = loose_start(c * BK + unit0, a.K), start1 = loose_start(c * BK + unit1, a.K);
#pragma unroll
            for (int i = 0; i < LOADS; ++i) to[i] = load_loose((i < 2 ? w0 : a.x) + row[i] + (i & 1 ? start1 : start0));
        };
        auto use = [&](u32x4 (&from)[LOADS], int c, int stage) {
            if ((c + 1) * BK > a.K) {
#pragma unroll
                for (int i = 2; i < LOADS; ++i) clear_counted(from[i], c * BK + (i & 1 ? unit1 : unit0), a.K);
            }
            char* const at = lds + (wave * STAGES + stage) * STAGE;
#pragma unroll
            for (int i = 0; i < LOADS; ++i) *reinterpret_cast<u32x4*>(at + i * 1024 + lane * 16) = from[i];
            load_loosely(from, c + STAGES * waves);
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            __builtin_amdgcn_wave_barrier();
            read(at);
            multiply();
        };
#pragma unroll
        for (int s = 0; s < STAGES; ++s) load_loosely(data[s], wave + s * waves);
        results.init(a, n0);
#pragma unroll 1
        for (int c = wave; c < chunks; c += STAGES * waves) {        // (chunks past the last one are cleared)
#pragma unroll
            for (int s = 0; s < STAGES; ++s) use(data[s], c + s * waves, s);
        }
    }
    wait_for_loads<0>();
    __syncthreads();
    int* const sums = reinterpret_cast<int*>(lds);
#pragma unroll
    for (int t = 0; t < TB; ++t)
#pragma unroll
        for (int e = 0; e < 4; ++e) sums[((wave * TB + t) * 4 + e) * 64 + lane] = acc[t][e];
    __syncthreads();
    results.store(a, sums, n0);
}

}  // namespace i8
}  // namespace anr
