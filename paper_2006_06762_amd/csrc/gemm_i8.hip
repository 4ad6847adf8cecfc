// Products of 8-bit integers with scales for rows and columns: which kernels a call runs.
//
//   few rows     i8_rows_kernel.h: reads the weights once
//   else         i8_tile_kernel.h; products with few tiles share each tile's k among work-groups, whose sums a second launch joins
#include <algorithm>

#include "blocks_internal.h"
#include "gemm_i8_plan.h"
#include "i8_rows_kernel.h"
#include "i8_tile_kernel.h"

namespace anr {
namespace {

using i8::Args;
using i8::Choice;
using i8::kChunk;
constexpr int kThreads = 256;

// D from the sums at `parts`, V columns a thread.
template <typename T, int V>
__global__ __launch_bounds__(kThreads) void join_kernel(const Args a, int units)
{
    const int64_t each = (int64_t)a.M * units, i = (int64_t)blockIdx.x * kThreads + threadIdx.x;
    if (i >= each) return;
    const int64_t m = each < (int64_t)1 << 31 ? (int64_t)((uint32_t)i / (uint32_t)units) : i / units;
    const int n = (int)(i - m * units) * V;
    Pack<int, V> sum = *reinterpret_cast<const Pack<int, V>*>(a.parts + i * V);
#pragma unroll 4
    for (int s = 1; s < a.splits; ++s) {
        const Pack<int, V> v = *reinterpret_cast<const Pack<int, V>*>(a.parts + (s * each + i) * V);
#pragma unroll
        for (int e = 0; e < V; ++e) sum.v[e] += v.v[e];
    }
    const float row = a.finish.of_row(m);
    float v[V];
#pragma unroll
    for (int e = 0; e < V; ++e) v[e] = i8::Finish::value(sum.v[e], row, a.finish.of_column(n + e), a.finish.added(n + e));
    store_floats<T, V>(static_cast<T*>(a.d) + m * a.ldd + n, v);
}

template <typename T>
hipError_t launch_join(const Args& a, hipStream_t stream)
{
    auto with = [&](auto v) {
        constexpr int V = decltype(v)::value;
        const int64_t groups = ((int64_t)a.M * (a.N / V) + kThreads - 1) / kThreads;
        return launch_kernel(join_kernel<T, V>, dim3((unsigned)groups), dim3(kThreads), 0, stream, a, a.N / V);
    };
    if (a.N % 4 == 0 && a.ldd % 4 == 0 && reinterpret_cast<uintptr_t>(a.d) % (4 * sizeof(T)) == 0) return with(std::integral_constant<int, 4>{});
    return with(std::integral_constant<int, 1>{});
}

// ---- few rows

template <typename T, int TB>
hipError_t launch_rows_as(const Args& a, bool loose, hipStream_t stream)
{
    constexpr int STAGES = 2;
    static LdsLimit limits[2];                   // of the two kernels
    const int waves = i8::waves_of(a.N, a.K, i8::most_waves(TB));
    void (*const kernel)(Args) = loose ? i8::stream_kernel<T, TB, STAGES, true> : i8::stream_kernel<T, TB, STAGES, false>;
    const size_t lds = std::max((size_t)waves * TB * 256 * sizeof(int), (size_t)waves * STAGES * (loose ? i8::stage_bytes<TB, true>() : i8::stage_bytes<TB, false>()));
    const hipError_t e = lds > 65536 ? raise_lds_limit(reinterpret_cast<const void*>(kernel), lds, limits[loose]) : hipSuccess;
    return e != hipSuccess ? e : launch_kernel(kernel, dim3((unsigned)((a.N + 15) / 16)), dim3(64 * waves), lds, stream, a);
}
template <typename T>
hipError_t launch_rows(const Args& a, bool loose, hipStream_t stream)
{
    if (a.M <= 16) return launch_rows_as<T, 1>(a, loose, stream);
    if (a.M <= 32) return launch_rows_as<T, 2>(a, loose, stream);
    return a.M <= 48 ? launch_rows_as<T, 3>(a, loose, stream) : launch_rows_as<T, 4>(a, loose, stream);
}

// ---- tiles

template <typename T, bool LOOSE, int M, int N, int WM, int WN, int STAGES>
hipError_t launch_as(Args a, hipStream_t stream)
{
    static LdsLimit limit;
    void (*const kernel)(Args) = i8::tile_kernel<T, M, N, WM, WN, kChunk, STAGES, LOOSE>;
    constexpr size_t lds = i8::tile_bytes<M, N, WM * WN, STAGES, LOOSE>();
    const hipError_t e = raise_lds_limit(reinterpret_cast<const void*>(kernel), lds, limit);
    if (e != hipSuccess) return e;
    a.tiles_m = (a.M + M - 1) / M;
    a.tiles_n = (a.N + N - 1) / N;
    a.band = 8;
    constexpr int LINE = 128 / (int)sizeof(T);
    a.streaming = N / WN % LINE == 0 && a.ldd % LINE == 0 && reinterpret_cast<uintptr_t>(a.d) % 128 == 0;
    return launch_kernel(kernel, dim3((unsigned)(a.tiles_m * a.tiles_n * a.splits)), dim3(64 * WM * WN), lds, stream, a);
}
template <typename T, bool LOOSE>
hipError_t launch_tile(int tile, const Args& a, hipStream_t stream)
{
    switch (tile) {
        case i8::TILE_256: return launch_as<T, LOOSE, 256, 256, 2, 4, 2>(a, stream);
        case i8::TILE_128: return launch_as<T, LOOSE, 128, 128, 2, 2, 2>(a, stream);
        case i8::TILE_128_DEEP: return launch_as<T, LOOSE, 128, 128, 2, 2, 3>(a, stream);
        case i8::TILE_64_128: return launch_as<T, LOOSE, 64, 128, 2, 2, 3>(a, stream);
        case i8::TILE_64: return launch_as<T, LOOSE, 64, 64, 2, 2, 3>(a, stream);
        default: return launch_as<T, LOOSE, 64, 64, 2, 2, 4>(a, stream);
    }
}

Choice choice_of(const anr_gemm_i8_desc& d)
{
    if (d.M == 0) return {i8::ROWS, 1};
    return i8::choose(d.M, d.N, d.K);
}

}  // namespace

size_t gemm_i8_workspace_bytes(const GemmI8Args& g)
{
    const int s = choice_of(g.d).splits;
    return s > 1 ? (size_t)s * g.d.M * g.d.N * sizeof(int) : 0;
}

hipError_t launch_gemm_i8(const GemmI8Args& g, hipStream_t stream)
{
    const anr_gemm_i8_desc& d = g.d;
    if (d.M == 0) return hipSuccess;
    Args a{};
    a.x = g.a;
    a.w = g.w;
    a.d = g.out;
    a.ldx = d.lda;
    a.ldw = d.ldw;
    a.ldd = d.ldd;
    a.M = (int)d.M;
    a.N = (int)d.N;
    a.K = (int)d.K;
    a.finish = {g.a_scale, g.w_scale, g.bias, d.bias_dtype};
    const Choice choice = choice_of(d);
    a.splits = choice.splits;
    a.parts = static_cast<int*>(g.ws);
    const bool loose = reinterpret_cast<uintptr_t>(g.a) % 4 != 0 || reinterpret_cast<uintptr_t>(g.w) % 4 != 0 || d.lda % 4 != 0 || d.ldw % 4 != 0;
    return with_type(d.dtype, [&](auto t) {
        using T = decltype(t);
        if (choice.tile == i8::ROWS) return launch_rows<T>(a, loose, stream);
        if (a.splits == 1) return loose ? launch_tile<T, true>(choice.tile, a, stream) : launch_tile<T, false>(choice.tile, a, stream);
        const hipError_t e = loose ? launch_tile<int, true>(choice.tile, a, stream) : launch_tile<int, false>(choice.tile, a, stream);
        return e != hipSuccess ? e : launch_join<T>(a, stream);
    });
}

}  // namespace anr
