// Products of a few rows X [M,K], M <= 16 TB, of 8-bit integers with a large matrix W (i8_device.h), as single tokens need them.
//
// Bound: reading W once.  A work-group takes 16 rows of W, its waves share the k in chunks of 128 and join their sums in LDS; the matrix instructions
// (v_mfma_i32_16x16x64_i8) are sixteen tokens wide, which cost nothing here.
#pragma once
#include "i8_device.h"

namespace anr {
namespace i8 {

constexpr int kRowsChunk = 128;                 // k of a wave at a time: a line of a row

// Sixteen values of k of a row that starts `row` bytes behind the base.
template <bool CLEAR>
__device__ __forceinline__ i32x4 load_unit(const int8_t* base, uint32_t row, int k, int K)
{
    u32x4 v = load_loose(base + row + loose_start(k, K));
    if (CLEAR) clear_counted(v, k, K);
    return __builtin_bit_cast(i32x4, v);
}

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

// Rows at any address and of any length from 16 on: from memory straight into the operands.  U: chunks of a wave whose loads are on their way together.
template <typename T, int TB, int U>
__global__ __launch_bounds__(1024) void rows_kernel(const Args a)
{
    extern __shared__ __attribute__((aligned(16))) int sums[];         // [wave][TB][4][64]
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), waves = blockDim.x >> 6;
    const int n0 = blockIdx.x * 16, r = lane & 15, g = lane >> 4;
    Results<T, TB> results;
    results.init(a, n0);
    const int8_t* const w0 = a.w + n0 * a.ldw;
    const uint32_t wrow = (uint32_t)(min(r, a.N - 1 - n0) * a.ldw);
    uint32_t xrow[TB];
#pragma unroll
    for (int t = 0; t < TB; ++t) xrow[t] = (uint32_t)(min(t * 16 + r, a.M - 1) * a.ldx);
    i32x4 acc[TB];
#pragma unroll
    for (int t = 0; t < TB; ++t) acc[t] = i32x4{0, 0, 0, 0};
    const int chunks = (a.K + kRowsChunk - 1) / kRowsChunk;
    for (int c = wave; c < chunks; c += waves * U) {
        i32x4 w[U][2], x[U][TB][2];
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const int k = (c + u * waves) * kRowsChunk + (4 * i + g) * kUnit;
                w[u][i] = load_unit<false>(w0, wrow, k, a.K);
#pragma unroll
                for (int t = 0; t < TB; ++t) x[u][t][i] = load_unit<true>(a.x, xrow[t], k, a.K);
            }
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int t = 0; t < TB; ++t) acc[t] = __builtin_amdgcn_mfma_i32_16x16x64_i8(w[u][i], x[u][t][i], acc[t], 0, 0, 0);
    }
#pragma unroll
    for (int t = 0; t < TB; ++t)
#pragma unroll
        for (int e = 0; e < 4; ++e) sums[((wave * TB + t) * 4 + e) * 64 + lane] = acc[t][e];
    __syncthreads();
    results.store(a, sums, n0);
}

// Rows of whole 16-byte units go through LDS: a lane's operand is of one of sixteen rows, and loads whose neighbouring lanes are in different lines take four times as
// long to issue (32 tokens 4096 -> 11264 19.4 us straight from memory, so 13.6; 1 token 5632 -> 2048 5.4, 4.1).  Each wave has STAGES buffers of its own, of its 16 rows of W and the 16 TB rows of X, and waits for no other one but at the end.
template <typename T, int TB, int STAGES>
__global__ __launch_bounds__(1024) void stream_kernel(const Args a)
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
#pragma unroll
    for (int s = 0; s < STAGES; ++s) load(wave + s * waves, s);
    Results<T, TB> results;
    results.init(a, n0);
    int stage = 0;
#pragma unroll 1
    for (int c = wave; c < chunks; c += waves) {
        wait_for_loads<(STAGES - 1) * LOADS>();
        const char* const at = lds + (wave * STAGES + stage) * STAGE;
        i32x4 v[2][1 + TB];
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int j = 0; j < 1 + TB; ++j) {
                const int r = lane & 15;
                v[i][j] = *reinterpret_cast<const i32x4*>(at + (j * 16 + r) * BK + place_of<BK>(r, 4 * i + (lane >> 4)) * kUnit);
            }
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
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int t = 0; t < TB; ++t) acc[t] = __builtin_amdgcn_mfma_i32_16x16x64_i8(v[i][0], v[i][1 + t], acc[t], 0, 0, 0);
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
