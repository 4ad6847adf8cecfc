// Products of 8-bit integers with scales for rows and columns: which kernels a call runs.
//
//   few rows     i8_rows_kernel.h: reads the weights once
//   else         i8_tile_kernel.h; products with few tiles share each tile's k among work-groups, whose sums a second launch joins
//   k below 16   one thread a result
#include <algorithm>

#include "blocks_internal.h"
#include "i8_rows_kernel.h"
#include "i8_tile_kernel.h"

namespace anr {
namespace {

using i8::Args;
constexpr int kThreads = 256;

template <typename T>
__global__ __launch_bounds__(kThreads) void short_kernel(const Args a)
{
    const int n = blockIdx.x * kThreads + threadIdx.x;
    if (n >= a.N) return;
    int w[i8::kUnit];
    for (int k = 0; k < a.K; ++k) w[k] = a.w[n * a.ldw + k];
    const float column = a.finish.of_column(n), added = a.finish.added(n);
    for (int m = blockIdx.y; m < a.M; m += gridDim.y) {
        int sum = 0;
        for (int k = 0; k < a.K; ++k) sum += a.x[m * a.ldx + k] * w[k];
        static_cast<T*>(a.d)[m * a.ldd + n] = from_float<T>(i8::Finish::value(sum, a.finish.of_row(m), column, added));
    }
}

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

constexpr bool few_rows(int64_t M) { return M <= 32; }

template <typename T, int TB, bool WHOLE>
hipError_t launch_rows_as(const Args& a, hipStream_t stream)
{
    static LdsLimit limit;
    // waves of a work-group: eight for each CU over all work-groups, as far as there are chunks for them
    const int groups = (a.N + 15) / 16, chunks = (a.K + i8::BK - 1) / i8::BK;
    int waves = 2;
    while (waves < 16 && groups * waves < 2048 && 2 * waves <= chunks) waves *= 2;
    const size_t lds = (size_t)waves * TB * 256 * sizeof(int);
    auto* const kernel = i8::rows_kernel<T, TB, WHOLE>;
    const hipError_t e = lds > 65536 ? raise_lds_limit(reinterpret_cast<const void*>(kernel), lds, limit) : hipSuccess;
    return e != hipSuccess ? e : launch_kernel(kernel, dim3(groups), dim3(64 * waves), lds, stream, a);
}
template <typename T>
hipError_t launch_rows(const Args& a, bool whole, hipStream_t stream)
{
    if (a.M <= 16) return whole ? launch_rows_as<T, 1, true>(a, stream) : launch_rows_as<T, 1, false>(a, stream);
    return whole ? launch_rows_as<T, 2, true>(a, stream) : launch_rows_as<T, 2, false>(a, stream);
}

// ---- tiles

enum Shape { SHAPE_256, SHAPE_128, SHAPE_128_TWICE };
int64_t tiles_of(int64_t M, int64_t N, int edge) { return ((M + edge - 1) / edge) * ((N + edge - 1) / edge); }
int64_t chunks_of(int64_t K) { return (K + i8::BK - 1) / i8::BK; }

// The tile with the shortest estimated time: rounds of work-groups over the CUs, each with its chunks and ends (us). A tile of 256 takes a CU
// for itself, of those of 128 it takes two; one alone is split over two groups of waves.
struct Choice {
    Shape shape;
    double us;
};
Choice choose_shape(int64_t tiles256, int64_t tiles128, int64_t chunks)
{
    const double large = (double)((tiles256 + 255) / 256) * (1.7 * (double)chunks + 4.0);
    const int64_t full = tiles128 / 512, rest = tiles128 % 512;
    const double pair = 1.14 * (double)chunks + 4.0, alone = 0.60 * (double)chunks + 4.0;
    const bool twice = tiles128 <= 256;
    const double small = twice ? alone : (double)full * pair + (rest > 256 ? pair : rest > 0 ? 0.75 * (double)chunks + 4.0 : 0.0);
    if (large < small) return {SHAPE_256, large};
    return {twice ? SHAPE_128_TWICE : SHAPE_128, small};
}

// Work-groups that share a tile's k, for products with few tiles: the number with the shortest estimated time, that of the launch that joins their
// sums among it. A function of the extents alone.
int splits_of(int64_t M, int64_t N, int64_t chunks)
{
    int best = 1;
    double least = choose_shape(tiles_of(M, N, 256), tiles_of(M, N, 128), chunks).us;
    for (int s = 2; s <= 16 && chunks / s >= 4; ++s) {
        const double us = choose_shape(s * tiles_of(M, N, 256), s * tiles_of(M, N, 128), (chunks + s - 1) / s).us + 4.0 + 2.0 * s * (double)M * (double)N * 4.0 / 8e6;
        if (us < least) {
            least = us;
            best = s;
        }
    }
    return best;
}

template <typename T, int BM, int BN, int WM, int WN, int G, bool WHOLE>
hipError_t launch_tile(Args a, hipStream_t stream)
{
    static LdsLimit limit;
    auto* const kernel = i8::tile_kernel<T, BM, BN, WM, WN, G, WHOLE>;
    constexpr size_t lds = G * i8::lds_bytes<BM, BN>();
    const hipError_t e = raise_lds_limit(reinterpret_cast<const void*>(kernel), lds, limit);
    if (e != hipSuccess) return e;
    a.tiles_m = (a.M + BM - 1) / BM;
    a.tiles_n = (a.N + BN - 1) / BN;
    a.band = 8;
    return launch_kernel(kernel, dim3((unsigned)(a.tiles_m * a.tiles_n * a.splits)), dim3(64 * WM * WN * G), lds, stream, a);
}
template <typename T>
hipError_t launch_shape(Shape shape, bool whole, const Args& a, hipStream_t stream)
{
    if (shape == SHAPE_256) return whole ? launch_tile<T, 256, 256, 2, 2, 1, true>(a, stream) : launch_tile<T, 256, 256, 2, 2, 1, false>(a, stream);
    if (shape == SHAPE_128) return whole ? launch_tile<T, 128, 128, 2, 2, 1, true>(a, stream) : launch_tile<T, 128, 128, 2, 2, 1, false>(a, stream);
    return whole ? launch_tile<T, 128, 128, 2, 2, 2, true>(a, stream) : launch_tile<T, 128, 128, 2, 2, 2, false>(a, stream);
}

int splits(const anr_gemm_i8_desc& d)
{
    if (d.M == 0 || d.K < i8::kUnit || few_rows(d.M)) return 1;
    return splits_of(d.M, d.N, chunks_of(d.K));
}

}  // namespace

size_t gemm_i8_workspace_bytes(const GemmI8Args& g)
{
    const int s = splits(g.d);
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
    a.splits = splits(d);
    a.parts = static_cast<int*>(g.ws);
    const bool whole = is_aligned16(g.a) && is_aligned16(g.w) && d.lda % 16 == 0 && d.ldw % 16 == 0 && d.K % 16 == 0;
    const int64_t chunks = chunks_of(d.K);
    return with_type(d.dtype, [&](auto t) {
        using T = decltype(t);
        if (d.K < i8::kUnit) {
            const int64_t columns = (d.N + kThreads - 1) / kThreads;     // (a grid has fewer than 2^32 threads)
            return launch_kernel(short_kernel<T>, dim3((unsigned)columns, (unsigned)std::min<int64_t>({d.M, 65535, (1 << 23) / columns})), dim3(kThreads), 0, stream, a);
        }
        if (few_rows(d.M)) return launch_rows<T>(a, whole, stream);
        const Shape shape = choose_shape(a.splits * tiles_of(d.M, d.N, 256), a.splits * tiles_of(d.M, d.N, 128), chunks / a.splits).shape;
        if (a.splits == 1) return launch_shape<T>(shape, whole, a, stream);
        const hipError_t e = launch_shape<int>(shape, whole, a, stream);
        return e != hipSuccess ? e : launch_join<T>(a, stream);
    });
}

}  // namespace anr
