// Products of a few rows X [T,K], T <= 16 TB, with a large matrix W [N,K] (rows of k), as single tokens need them:
// D[t][n] = sum_k X[t][k] W[n][k], and for the gated block the same with two matrices and act(g) u of their sums.
//
// Bound: reading W once.  A work-group takes 16 rows of W (of both matrices), its waves share the k in chunks of 128 bytes
// a row and join their sums in LDS; W goes from memory straight into the operands of the matrix instructions, sixteen tokens wide
// (which cost nothing here), without LDS: nothing of it is used twice.  A lane's part of a chunk are two units of a row, so
// the order of k differs from memory's, in both operands alike.
#pragma once
#include "anr_kernels.h"
#include "element_types.h"
#include "mm16_kernel.h"

namespace anr {
namespace ffrows {

using mm16::f16x8;
using mm16::b16x8;
using mm16::kExtent;
using mm16::kNowhere;
using mm16::u32x4;

struct Args {
    const void* x;
    const void* w[2];               // rows: the one matrix; gated: gate's and up's
    void* d;
    void *gate, *up;                // gated: where the sums go, or null
    int64_t ldx, ldw[2], ldd, ld_pre;
    int T, N, K;
    int act;
    bool whole_rows;                // gated: D's rows go on in zeros to the end of their last 16 bytes
};

// Sixteen bytes of each operand.
__device__ __forceinline__ f32x4 multiply(u32x4 w, u32x4 x, f32x4 c, half_t)
{
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, w), __builtin_bit_cast(f16x8, x), c, 0, 0, 0);
}
__device__ __forceinline__ f32x4 multiply(u32x4 w, u32x4 x, f32x4 c, bf16_t)
{
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(b16x8, w), __builtin_bit_cast(b16x8, x), c, 0, 0, 0);
}
__device__ __forceinline__ f32x4 multiply(u32x4 w, u32x4 x, f32x4 c, float)
{
    const f32x4 a = __builtin_bit_cast(f32x4, w), b = __builtin_bit_cast(f32x4, x);
#pragma unroll
    for (int i = 0; i < 4; ++i) c = mfma16(a[i], b[i], c);
    return c;
}

// A matrix that a lane reads rows of.
struct Source {
    const char* base;
    __amdgpu_buffer_rsrc_t rsrc;
    __device__ __forceinline__ void init(const void* p)
    {
        base = static_cast<const char*>(p);
        rsrc = __builtin_amdgcn_make_buffer_rsrc(const_cast<char*>(base), 0, kExtent, 0x00020000);
    }
};

// Elements k .. k + 16 / sizeof(T) - 1 of the row at byte `row` of a matrix; those past K are zeros.  ALIGNED: pointers, leading dimensions
// and K are whole 16-byte units, but for rows that go on in zeros to the end of their last one.  Else a row's last unit starts so far ahead that
// it ends with the row, and what the unit before it has is cleared: other elements of k in its place, in both operands alike.
template <typename T, bool ALIGNED>
__device__ __forceinline__ u32x4 load_unit(const Source& s, uint32_t row, int k, int K)
{
    constexpr int E = 16 / sizeof(T);
    if (ALIGNED) return __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(s.rsrc, (int)(k < K ? row + k * (int)sizeof(T) : kNowhere), 0, 0));
    u32x4 v = {0, 0, 0, 0};
    if (K >= E) {
        struct __attribute__((packed, aligned(2))) Loose { u32x4 v; };
        const int start = min(k, K - E), counted = k < K ? k - start : E;
        v = reinterpret_cast<const Loose*>(s.base + row + start * (int)sizeof(T))->v;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            if (sizeof(T) == 4) v[j] = j < counted ? 0u : v[j];
            else v[j] &= (2 * j < counted ? 0u : 0x0000ffffu) | (2 * j + 1 < counted ? 0u : 0xffff0000u);
        }
        return v;
    }
#pragma unroll
    for (int j = 0; j < E; ++j) {
        const int at = (int)(k + j < K ? row + (k + j) * (int)sizeof(T) : kNowhere);
        if (sizeof(T) == 4) v[j * (int)sizeof(T) / 4] = __builtin_amdgcn_raw_buffer_load_b32(s.rsrc, at, 0, 0);
        else v[j / 2] |= (uint32_t)(uint16_t)__builtin_amdgcn_raw_buffer_load_b16(s.rsrc, at, 0, 0) << (16 * (j & 1));
    }
    return v;
}

template <typename T, int TB, bool GATED, bool ALIGNED>
__global__ __launch_bounds__(1024) void rows_kernel(const Args a)
{
    constexpr int E = 16 / sizeof(T), CHUNK = 128 / sizeof(T), MATS = GATED ? 2 : 1;
    constexpr int U = TB == 1 ? 3 : TB == 2 ? 2 : 1;                   // chunks of a wave whose loads are on their way together
    extern __shared__ __attribute__((aligned(16))) float sums[];       // [wave][TB][MATS][4][64]
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), waves = blockDim.x >> 6;
    const int n0 = blockIdx.x * 16, r = lane & 15, g = lane >> 4;
    Source wr[MATS], xr;
    uint32_t wrow[MATS], xrow[TB];
#pragma unroll
    for (int m = 0; m < MATS; ++m) {
        wr[m].init(static_cast<const T*>(a.w[m]) + n0 * a.ldw[m]);
        wrow[m] = (uint32_t)(min(r, a.N - 1 - n0) * a.ldw[m] * sizeof(T));
    }
    xr.init(a.x);
#pragma unroll
    for (int t = 0; t < TB; ++t) xrow[t] = (uint32_t)(min(t * 16 + r, a.T - 1) * a.ldx * sizeof(T));
    f32x4 acc[MATS][TB];
#pragma unroll
    for (int m = 0; m < MATS; ++m)
#pragma unroll
        for (int t = 0; t < TB; ++t) acc[m][t] = zero4();
    const int chunks = (a.K + CHUNK - 1) / CHUNK;
    for (int c = wave; c < chunks; c += waves * U) {
        u32x4 w[U][MATS][2], x[U][TB][2];
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const int k = (c + u * waves) * CHUNK + (4 * i + g) * E;
#pragma unroll
                for (int m = 0; m < MATS; ++m) w[u][m][i] = load_unit<T, ALIGNED>(wr[m], wrow[m], k, a.K);
#pragma unroll
                for (int t = 0; t < TB; ++t) x[u][t][i] = load_unit<T, ALIGNED>(xr, xrow[t], k, a.K);
            }
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int m = 0; m < MATS; ++m)
#pragma unroll
                    for (int t = 0; t < TB; ++t) acc[m][t] = multiply(w[u][m][i], x[u][t][i], acc[m][t], T{});
    }
#pragma unroll
    for (int t = 0; t < TB; ++t)
#pragma unroll
        for (int m = 0; m < MATS; ++m)
#pragma unroll
            for (int e = 0; e < 4; ++e) sums[(((wave * TB + t) * MATS + m) * 4 + e) * 64 + lane] = acc[m][t][e];
    __syncthreads();
    // register e of lane l: row 4 (l / 16) + e of W, token l % 16
    for (int i = tid; i < TB * 256; i += (int)blockDim.x) {
        const int t = i >> 8, e = (i >> 6) & 3, l = i & 63, token = t * 16 + (l & 15), n = n0 + 4 * (l >> 4) + e;
        float v[MATS];
#pragma unroll
        for (int m = 0; m < MATS; ++m) {
            v[m] = 0.f;
            for (int w = 0; w < waves; ++w) v[m] += sums[(((w * TB + t) * MATS + m) * 4 + e) * 64 + l];
        }
        constexpr int UNIT = 16 / sizeof(T);
        if (GATED && a.whole_rows && token < a.T && n >= a.N && n < (a.N + UNIT - 1) / UNIT * UNIT) static_cast<T*>(a.d)[token * a.ldd + n] = from_float<T>(0.f);
        if (token >= a.T || n >= a.N) continue;
        float out = v[0];
        if (GATED) {
            if (a.gate) {
                static_cast<T*>(a.gate)[token * a.ld_pre + n] = from_float<T>(v[0]);
                static_cast<T*>(a.up)[token * a.ld_pre + n] = from_float<T>(v[MATS - 1]);
            }
            device_activation(a.act, [&](auto act) { out = activation<decltype(act)::value, sizeof(T) == 2>(v[0]) * v[MATS - 1]; });
        }
        static_cast<T*>(a.d)[token * a.ldd + n] = from_float<T>(out);          // (gated: h, in the type that the next product's instructions take)
    }
}

}  // namespace ffrows
}  // namespace anr
