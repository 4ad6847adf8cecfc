// Products of a few rows X [M,K], M <= 16 TB, of 8-bit integers with a large matrix W (i8_device.h), as single tokens need them.
//
// Bound: reading W once.  A work-group takes 16 rows of W, its waves share the k in chunks of 128 and join their sums in LDS; W goes from
// memory straight into the operands of the matrix instructions (v_mfma_i32_16x16x64_i8), sixteen tokens wide (which cost nothing here), without
// LDS: nothing of it is used twice.
#pragma once
#include "i8_device.h"

namespace anr {
namespace i8 {

constexpr int kRowsChunk = 128;                 // k of a wave at a time: a line of a row

// Sixteen values of k of a row that starts `row` bytes behind the base.
template <bool WHOLE, bool CLEAR>
__device__ __forceinline__ i32x4 load_unit(const int8_t* base, uint32_t row, int k, int K)
{
    u32x4 v;
    if (WHOLE) {
        const __amdgpu_buffer_rsrc_t rsrc = __builtin_amdgcn_make_buffer_rsrc(const_cast<int8_t*>(base), 0, kExtent, 0x00020000);
        v = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(rsrc, (int)(k < K ? row + k : kNowhere), 0, 0));
    } else {
        v = load_loose(base + row + loose_start(k, K));
        if (CLEAR) clear_counted(v, k, K);
    }
    return __builtin_bit_cast(i32x4, v);
}

template <typename T, int TB, bool WHOLE>
__global__ __launch_bounds__(1024) void rows_kernel(const Args a)
{
    constexpr int U = TB == 1 ? 3 : TB == 2 ? 2 : 1;                   // chunks of a wave whose loads are on their way together
    extern __shared__ __attribute__((aligned(16))) int sums[];         // [wave][TB][4][64]
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), waves = blockDim.x >> 6;
    const int n0 = blockIdx.x * 16, r = lane & 15, g = lane >> 4;
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
                w[u][i] = load_unit<WHOLE, false>(w0, wrow, k, a.K);
#pragma unroll
                for (int t = 0; t < TB; ++t) x[u][t][i] = load_unit<WHOLE, true>(a.x, xrow[t], k, a.K);
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
    // register e of lane l: row 4 (l / 16) + e of W, token l % 16
    for (int i = tid; i < TB * 256; i += (int)blockDim.x) {
        const int t = i >> 8, e = (i >> 6) & 3, l = i & 63, token = t * 16 + (l & 15), n = n0 + 4 * (l >> 4) + e;
        if (token >= a.M || n >= a.N) continue;
        int v = 0;
        for (int w = 0; w < waves; ++w) v += sums[((w * TB + t) * 4 + e) * 64 + l];
        static_cast<T*>(a.d)[token * a.ldd + n] = from_float<T>(Finish::value(v, a.finish.of_row(token), a.finish.of_column(n), a.finish.added(n)));
    }
}

}  // namespace i8
}  // namespace anr
