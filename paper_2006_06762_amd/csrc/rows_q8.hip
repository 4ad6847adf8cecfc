// Rows of values to 8 bits with a scale each, and back (rows_device.h).
//
// v = act(x) up is formed once, held in the registers of the waves that have the row while its largest magnitude is found, and stored in steps of a 127th of that:
// memory is read once.  Rows of more than 32768 values are formed twice.
#include <algorithm>

#include "blocks_internal.h"
#include "rows_device.h"
#include "rows_launch.h"

namespace anr {
namespace {

using namespace rows;

constexpr int kMostGroups = 1 << 20;             // of a launch: rows beyond them are taken in turn
constexpr int kLongThreads = 1024;
constexpr int kBackThreads = 256;

struct Args {
    const void *x, *up;
    int8_t* q;
    float* scale;
    int64_t T, ldx, ld_up, ldq;
    int C, act;
};

// v = act(x) up, in place of x.
template <int ACT, bool QUICK, int V>
__device__ __forceinline__ void gate(float (&x)[V], const float (&up)[V], bool gated)
{
#pragma unroll
    for (int j = 0; j < V; ++j) {
        x[j] = activation<ACT, QUICK>(x[j]);
        if (gated) x[j] *= up[j];
    }
}

template <typename T, int V, int U, bool WHOLE>
__global__ __launch_bounds__(1024) void quantize_kernel(const Args a)
{
    const int threads = blockDim.x, t = threadIdx.x, C = a.C;
    int round = 0;
    for (int64_t first = (int64_t)blockIdx.x * blockDim.y; first < a.T; first += (int64_t)gridDim.x * blockDim.y, round ^= 1) {
        const int64_t row = row_of<(U > 2)>(first + threadIdx.y < a.T ? first + threadIdx.y : a.T - 1);      // (rows past the end repeat the last one and store nothing)
        const bool in = first + threadIdx.y < a.T;
        Raw<T, V> x[U], up[U];
#pragma unroll
        for (int u = 0; u < U; ++u) x[u].load(static_cast<const T*>(a.x) + row * a.ldx + Unit<V, WHOLE>(t + u * threads, C).start);
        if (a.up) {
#pragma unroll
            for (int u = 0; u < U; ++u) up[u].load(static_cast<const T*>(a.up) + row * a.ld_up + Unit<V, WHOLE>(t + u * threads, C).start);
        }
        float v[U][V];
        Joined of{0.f, 0u};
        // (a branch for each unit: all of them in one block's registers spilled 1200 bytes a thread, and 8192 x 11264 gated took 2200 us)
#pragma unroll
        for (int u = 0; u < U; ++u) {
            float w[V];
            x[u].floats(v[u]);
            if (a.up) up[u].floats(w);
            device_activation(a.act, [&](auto act) { gate<decltype(act)::value, sizeof(T) == 2>(v[u], w, a.up != nullptr); });
#pragma unroll
            for (int j = 0; j < V; ++j) of.largest = max(of.largest, magnitude(v[u][j]));
        }
        of = join_row<false, true>(of, round);
        if (!in) continue;
        const Steps steps(of.largest, 1.f);
        if (t == 0) a.scale[row] = steps.step;
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const Unit<V, WHOLE> unit(t + u * threads, C);
            if (unit.in()) store_steps<V>(a.q + row * a.ldq + unit.start, v[u], steps);
        }
    }
}

// Rows that no work-group holds.
template <typename T, int V>
__global__ __launch_bounds__(kLongThreads) void quantize_long_kernel(const Args a)
{
    const int C = a.C;
    int round = 0;
    for (int64_t row = blockIdx.x; row < a.T; row += gridDim.x, round ^= 1) {
        device_activation(a.act, [&](auto act) {
            auto form = [&](const Unit<V, false>& unit, float (&v)[V]) {
                Raw<T, V> x, up;
                float w[V];
                x.load(static_cast<const T*>(a.x) + row * a.ldx + unit.start);
                x.floats(v);
                if (a.up) {
                    up.load(static_cast<const T*>(a.up) + row * a.ld_up + unit.start);
                    up.floats(w);
                }
                gate<decltype(act)::value, sizeof(T) == 2>(v, w, a.up != nullptr);
            };
            Joined of{0.f, 0u};
            float v[V];
            for (int i = threadIdx.x; i * V < C; i += kLongThreads) {
                form(Unit<V, false>(i, C), v);
#pragma unroll
                for (int j = 0; j < V; ++j) of.largest = max(of.largest, magnitude(v[j]));
            }
            of = join_row<false, true>(of, round);
            const Steps steps(of.largest, 1.f);
            if (threadIdx.x == 0) a.scale[row] = steps.step;
            for (int i = threadIdx.x; i * V < C; i += kLongThreads) {
                const Unit<V, false> unit(i, C);
                form(unit, v);
                store_steps<V>(a.q + row * a.ldq + unit.start, v, steps);
            }
        });
    }
}

struct BackArgs {
    const int8_t* q;
    const float* scale;
    void* y;
    int64_t T, ldq, ldy;
    int C;
};

template <typename T, int V>
__global__ __launch_bounds__(kBackThreads) void dequantize_kernel(const BackArgs a)
{
    struct __attribute__((packed, aligned(1))) Loose { int8_t v[V]; };
    const int i = blockIdx.x * blockDim.x + threadIdx.x;
    const Unit<V, false> unit(i, a.C);
    if (!unit.in()) return;
    for (int64_t row = (int64_t)blockIdx.y * blockDim.y + threadIdx.y; row < a.T; row += (int64_t)gridDim.y * blockDim.y) {
        const Loose l = *reinterpret_cast<const Loose*>(a.q + row * a.ldq + unit.start);
        const float scale = a.scale[row];
        float v[V];
#pragma unroll
        for (int j = 0; j < V; ++j) v[j] = (float)l.v[j] * scale;
        store<true>(static_cast<T*>(a.y) + row * a.ldy + unit.start, v);
    }
}

}  // namespace

hipError_t launch_quantize_rows(const RowsQ8Args& g, hipStream_t stream)
{
    if (g.d.T == 0) return hipSuccess;
    const Args a{g.x, g.up, g.q, g.scale, g.d.T, g.d.ldx, g.d.ld_up, g.d.ldq, (int)g.d.C, g.d.act};
    return with_type(g.d.dtype, [&](auto t) {
        using T = decltype(t);
        if (a.C > kHeldBy1024)
            return launch_kernel(quantize_long_kernel<T, 16 / (int)sizeof(T)>, dim3((unsigned)std::min<int64_t>(a.T, kMostGroups)), dim3(kLongThreads), 0, stream, a);
        const Plan of = plan_for<T>(a.C, a.T);
        return with_rows<T>(a.C, of, [&](auto v, auto u, auto whole) {
            const int64_t groups = std::min<int64_t>((a.T + of.rows - 1) / of.rows, kMostGroups);
            return launch_kernel(quantize_kernel<T, decltype(v)::value, decltype(u)::value, decltype(whole)::value>, dim3((unsigned)groups), dim3(of.threads, of.rows), 0, stream,
                                 a);
        });
    });
}

hipError_t launch_dequantize_rows(const RowsQ8Args& g, hipStream_t stream)
{
    if (g.d.T == 0) return hipSuccess;
    return with_type(g.d.dtype, [&](auto t) {
        using T = decltype(t);
        const int V = values_of<T>(g.d.C), units = (int)((g.d.C + V - 1) / V);
        const BackArgs a{g.q, g.scale, const_cast<void*>(g.x), g.d.T, g.d.ldq, g.d.ldx, (int)g.d.C};
        int wide = 1;                            // threads on a row, a power of two
        while (wide < kBackThreads && wide < units) wide *= 2;
        const int64_t rows = kBackThreads / wide;
        const int64_t columns = (units + wide - 1) / wide;               // (a grid has fewer than 2^32 threads)
        const dim3 grid((unsigned)columns, (unsigned)std::min<int64_t>({(g.d.T + rows - 1) / rows, 65535, (1 << 23) / columns})), block(wide, (unsigned)rows);
        if (V == 1) return launch_kernel(dequantize_kernel<T, 1>, grid, block, 0, stream, a);
        return launch_kernel(dequantize_kernel<T, 16 / (int)sizeof(T)>, grid, block, 0, stream, a);
    });
}

}  // namespace anr
