// Products of 8-bit integers with scales for rows and columns: which kernels a call runs.
//
//   few rows     i8_rows_kernel.h: reads the weights once
//   else         i8_tile_kernel.h; products with few tiles share each tile's k among work-groups, whose sums a second launch joins
#include <algorithm>

#include "blocks_internal.h"
#include "i8_rows_kernel.h"
#include "i8_tile_kernel.h"

namespace anr {
namespace {

using i8::Args;
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

// Waves of a work-group: as far as there are chunks for them, eight for each CU over all work-groups, or long rows. us, 4 / 8 / 16 waves: 1 token 2048 -> 11264
// 6.0 / 6.9 / 9.7, 5632 -> 2048 4.8 / 4.0 / 4.3, 1024 -> 1024 2.74 / 2.68 / 3.1, 16384 -> 16384 54.1 / 50.6 / 52.2, 8 tokens 4096 -> 4096 5.9 / 5.6 / 5.4.
int waves_of(int64_t N, int64_t K, int most)
{
    const int64_t groups = (N + 15) / 16, chunks = (K + i8::kRowsChunk - 1) / i8::kRowsChunk;
    int waves = 4;
    while (waves < most && chunks >= 4 * waves && (groups * waves <= 2048 || chunks >= 16 * waves)) waves *= 2;
    return waves;
}
template <typename T, int TB>
hipError_t launch_rows_as(const Args& a, bool loose, hipStream_t stream)
{
    constexpr int STAGES = 2;
    static LdsLimit limits[2];                   // of the two kernels
    const int waves = waves_of(a.N, a.K, i8::most_waves(TB));
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

constexpr int64_t kChunk = 128;                  // k of a chunk
constexpr int kCus = 256;

// A tile, how many of its work-groups a CU takes at a time, and its estimated time in us: a chunk's where a work-group is alone on its CU and where that is full, and that
// of both ends.  The deep ones have a chunk more on their way, for products of few tiles: 64 tokens 4096 -> 11264 in tiles of 64 with two, three and four buffers 17.7 / 11.3 / 10.4 us, 777 tokens 640 -> 1363
// 5.2 / 5.4 / 5.7; 256 tokens 4096 -> 11264 in tiles of 128 with two and three 24.1 / 16.9 and 512 tokens 27.9 / 32.1.
struct Shape {
    int m, n, on_cu;
    double alone, full, ends;
};
enum { TILE_256, TILE_128, TILE_128_DEEP, TILE_64_128, TILE_64, TILE_64_DEEP, TILES, ROWS = TILES };
constexpr Shape kShapes[TILES] = {
    {256, 256, 1, 1.18, 1.18, 4.5}, {128, 128, 2, 0.59, 0.69, 3.3}, {128, 128, 1, 0.35, 0.35, 4.6}, {64, 128, 2, 0.30, 0.50, 3.1}, {64, 64, 3, 0.22, 0.69, 2.9}, {64, 64, 2, 0.175, 0.46, 3.4}};

int64_t tiles_of(int64_t M, int64_t N, const Shape& s) { return ((M + s.m - 1) / s.m) * ((N + s.n - 1) / s.n); }

double estimate(const Shape& s, int64_t tiles, int64_t chunks)
{
    const int64_t at_once = (int64_t)s.on_cu * kCus, rounds = tiles / at_once, rest = tiles % at_once, beside = (rest + kCus - 1) / kCus;
    double us = (double)rounds * (s.full * (double)chunks + s.ends);
    if (rest > 0) us += (s.on_cu > 1 ? s.alone + (s.full - s.alone) * (double)(beside - 1) / (double)(s.on_cu - 1) : s.full) * (double)chunks + s.ends;
    return us;
}

// The kernels for few rows: reading W, and X for every sixteen of W's rows, and a round of the waves' chunks.
double estimate_rows(int64_t M, int64_t N, int64_t K)
{
    const int64_t groups = (N + 15) / 16, blocks = (M + 15) / 16, chunks = (K + kChunk - 1) / kChunk, waves = waves_of(N, K, i8::most_waves((int)blocks));
    return 3.0 + (double)N * (double)K / 11.1e6 + (double)(groups * blocks * 16) * (double)K / 71e6 + 0.078 * (double)((1 + blocks) * ((chunks + waves - 1) / waves));
}

// The tile, or the kernels for few rows, and the work-groups that share a tile's k where there are few, with the shortest estimated time, that of the launch that joins their
// sums among it.  A function of the extents alone.  The estimates' numbers are fitted to 272 products of 1 to 2048 rows, 256 -> 4096 to 4096 -> 16384, each by every tile and 1 to 8
// parts of k: what is chosen took 1 % longer than the fastest on average.
struct Choice {
    int tile, splits;
};
constexpr int64_t kMostRows = 64;
Choice choose(int64_t M, int64_t N, int64_t K)
{
    const int64_t chunks = (K + kChunk - 1) / kChunk;
    Choice best{ROWS, 1};
    double least = M <= kMostRows ? estimate_rows(M, N, K) : 1e30;
    for (int t = 0; t < TILES; ++t)
        for (int s = 1; s <= 16 && (s == 1 || chunks / s >= 4); ++s) {
            const double us = estimate(kShapes[t], s * tiles_of(M, N, kShapes[t]), (chunks + s - 1) / s) + (s > 1 ? 3.45 + 2.0 * s * (double)M * (double)N * 4.0 / 4.6e6 : 0.0);
            if (us < least) {
                least = us;
                best = {t, s};
            }
        }
    return best;
}

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
        case TILE_256: return launch_as<T, LOOSE, 256, 256, 2, 4, 2>(a, stream);
        case TILE_128: return launch_as<T, LOOSE, 128, 128, 2, 2, 2>(a, stream);
        case TILE_128_DEEP: return launch_as<T, LOOSE, 128, 128, 2, 2, 3>(a, stream);
        case TILE_64_128: return launch_as<T, LOOSE, 64, 128, 2, 2, 3>(a, stream);
        case TILE_64: return launch_as<T, LOOSE, 64, 64, 2, 2, 3>(a, stream);
        default: return launch_as<T, LOOSE, 64, 64, 2, 2, 4>(a, stream);
    }
}

Choice choice_of(const anr_gemm_i8_desc& d)
{
    if (d.M == 0) return {ROWS, 1};
    return choose(d.M, d.N, d.K);
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
        if (choice.tile == ROWS) return launch_rows<T>(a, loose, stream);
        if (a.splits == 1) return loose ? launch_tile<T, true>(choice.tile, a, stream) : launch_tile<T, false>(choice.tile, a, stream);
        const hipError_t e = loose ? launch_tile<int, true>(choice.tile, a, stream) : launch_tile<int, false>(choice.tile, a, stream);
        return e != hipSuccess ? e : launch_join<T>(a, stream);
    });
}

}  // namespace anr
