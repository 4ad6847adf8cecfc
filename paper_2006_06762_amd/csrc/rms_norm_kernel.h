// Root-mean-square norm of rows with the residual's addition, and its gradients.  h = x + residual, rstd = 1 / sqrt(mean(h^2) + eps),
// y = h rstd gamma: a row is read once, held in registers (rows_device.h) and summed by the waves that have it.
//
// In 8 bits the largest |y| of a row is rstd times that of |h gamma|, which is found with the sum of the squares in one go, and y is the same
// number of its steps as h gamma of its own.
//
// Backward, with dhat = dy gamma and hat = x rstd: dx = rstd (dhat - hat mean(dhat hat)) + dh, and dgamma = sum over the rows of dy hat.  A
// work-group goes over several rows and sums dgamma of its columns in registers; a second launch joins the work-groups' sums in their order.
#pragma once
#include "anr_kernels.h"
#include "rows_device.h"
#include "rows_plan.h"

namespace anr {
namespace rmsnorm {

struct Args {
    const void *x, *residual, *gamma;
    void *h, *y;                    // y: q where the output is in 8 bits
    float *rstd, *scale;
    float eps;
    int64_t T;
    int C;
    int64_t ldx, ld_residual, ldh, ldy;
    bool streaming;                 // outputs go past L2.  Of the call, not of the type: with the stores in the loop's own block the compiler converts the next row's values in front of them (8192 x 4096 bf16
                                    // backward 55 us, 60 so)
    // backward
    const void *dy, *dh;            // (dx goes to h)
    const float* rstd_in;
    float* sums;                    // [work-groups][C], or null: no dgamma
};

// Behind each unit of a thread that holds many: all units' values in one schedule spilled more.  (32 values a thread beside gamma's, forward, or dy, backward, still are more than 128 registers: 1024 x 32768 float32 with the
// residual 152 bytes of scratch a lane, 132 us for 105 by its bytes, backward with dh 192 and 188 us; bf16 normed to 8 bits 48 and 64.5 for 46, backward 80 and 86 for 52.)
template <int HELD>
__device__ __forceinline__ void unit_done()
{
    if (HELD >= 32) __builtin_amdgcn_sched_barrier(0);
}

// P: gamma's type.  U units of a thread.
template <typename T, typename P, int V, int U, bool WHOLE, bool QUANTIZED, int THREADS>
__global__ __launch_bounds__(THREADS) void forward_kernel(const Args a)
{
    using namespace rows;
    const int threads = blockDim.x, t = threadIdx.x, C = a.C;
    Raw<P, V> g[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
        if (a.gamma) g[u].load(static_cast<const P*>(a.gamma) + Unit<V, WHOLE>(t + u * threads, C).start);
        else g[u].fill(from_float<P>(1.f));
    }
    int round = 0;
    for (int64_t first = (int64_t)blockIdx.x * blockDim.y; first < a.T; first += (int64_t)gridDim.x * blockDim.y, round ^= 1) {
        const int64_t row = row_of<(U > 2)>(first + threadIdx.y < a.T ? first + threadIdx.y : a.T - 1);      // (rows past the end repeat the last one and store nothing)
        const bool in = first + threadIdx.y < a.T;
        Raw<T, V> x[U], r[U];
#pragma unroll
        for (int u = 0; u < U; ++u) x[u].load(static_cast<const T*>(a.x) + row * a.ldx + Unit<V, WHOLE>(t + u * threads, C).start);
        if (a.residual) {
#pragma unroll
            for (int u = 0; u < U; ++u) r[u].load(static_cast<const T*>(a.residual) + row * a.ld_residual + Unit<V, WHOLE>(t + u * threads, C).start);
        }
        float h[U][V];
        Joined of{0.f, 0u};
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const Unit<V, WHOLE> unit(t + u * threads, C);
            x[u].floats(h[u]);
            if (a.residual) {
                float v[V];
                r[u].floats(v);
#pragma unroll
                for (int j = 0; j < V; ++j) h[u][j] += v[j];
            }
            float gamma[V];
            if (QUANTIZED) g[u].floats(gamma);
            float sum = 0.f;
#pragma unroll
            for (int j = 0; j < V; ++j) {
                if (WHOLE || unit.counts(j)) sum = fmaf(h[u][j], h[u][j], sum);
                if (QUANTIZED) of.largest = max(of.largest, magnitude(h[u][j] * gamma[j]));
            }
            if (!WHOLE || unit.in()) of.sum += sum;
            unit_done<U * V>();
        }
        of = join_row<true, QUANTIZED>(of, round);
        const float rstd = 1.f / sqrtf(of.sum / (float)C + a.eps);
        if (!in) continue;
#pragma unroll
        for (int u = 0; u < U; ++u) g[u].keep_packed();
        const Steps steps(of.largest, rstd);
        if (t == 0) {
            if (a.rstd) a.rstd[row] = rstd;
            if (QUANTIZED) a.scale[row] = steps.step;
        }
        by_streaming(a.streaming, [&](auto streaming) {
            constexpr bool S = decltype(streaming)::value;
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const Unit<V, WHOLE> unit(t + u * threads, C);
                if (!unit.in()) continue;
                if (a.h) store<S>(static_cast<T*>(a.h) + row * a.ldh + unit.start, h[u]);
                float gamma[V], y[V];
                g[u].floats(gamma);
#pragma unroll
                for (int j = 0; j < V; ++j) y[j] = QUANTIZED ? h[u][j] * gamma[j] : h[u][j] * rstd * gamma[j];
                if (QUANTIZED) store_steps<V>(static_cast<int8_t*>(a.y) + row * a.ldy + unit.start, y, steps);
                else store<S>(static_cast<T*>(a.y) + row * a.ldy + unit.start, y);
                unit_done<U * V>();
            }
        });
    }
}

// What a row's gradients are made of.
template <typename T, int V, int U, bool WHOLE>
struct Row {
    rows::Raw<T, V> x[U], dy[U], dh[U];
    float rstd;
    __device__ __forceinline__ void load_dh(const Args& a, int64_t row, int t, int u)
    {
        dh[u].load(rows::at<T>(static_cast<const T*>(a.dh) + row * a.ld_residual, rows::Unit<V, WHOLE>(t + u * (int)blockDim.x, a.C).start));
    }
    __device__ __forceinline__ void load(const Args& a, int64_t row, int t, bool with_dh)
    {
        const int threads = blockDim.x, C = a.C;
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int start = rows::Unit<V, WHOLE>(t + u * threads, C).start;
            dy[u].load(rows::at<T>(static_cast<const T*>(a.dy) + row * a.ldy, start));
            x[u].load(rows::at<T>(static_cast<const T*>(a.x) + row * a.ldx, start));
        }
        if (with_dh && a.dh) {
#pragma unroll
            for (int u = 0; u < U; ++u) load_dh(a, row, t, u);
        }
        rstd = a.rstd_in[row];
    }
};

// Whether the sums of a thread with so many values lie in LDS, since its registers do not hold them too (1024 x 32768 bf16 149 us, so 71; with sums of 16 values there and the next row on its way instead 4096 x 8200
// 62, so 64).
constexpr bool sums_apart(int values) { return values > 16; }

// A row's values are on their way while those of the row before are used, as far as the registers hold both (bf16 8192 x 4096 with the gradient of the residual 61.5 us, so 57.8;
// two units of eight 57.1, so 65.6).
template <typename T, typename P, int V, int U, bool WHOLE, int THREADS>
__global__ __launch_bounds__(THREADS) void backward_kernel(const Args a)
{
    using namespace rows;
    extern __shared__ __attribute__((aligned(16))) float shared[];   // sums of the rows of a work-group that has several, [rows][C]; or a thread's sums, [unit][V / 4][kMostThreads][4]
    const int threads = blockDim.x, t = threadIdx.x, C = a.C;
    constexpr bool FEW = U * V <= 8;             // values of a thread: more, and gamma and dh are read where they are used
    constexpr bool APART = sums_apart(U * V), FORMED = U > 2;
    Raw<P, V> g[U];
    float sums[APART ? 1 : U][V];
    auto load_gamma = [&](int t, int u) {
        if (a.gamma) g[u].load(at<P>(a.gamma, Unit<V, WHOLE>(t + u * threads, C).start));
        else g[u].fill(from_float<P>(1.f));
    };
#pragma unroll
    for (int u = 0; u < U; ++u) {
        if (FEW) load_gamma(t, u);
        if (APART) {
#pragma unroll
            for (int j = 0; j < V; j += 4) *reinterpret_cast<f32x4*>(shared + ((u * V + j) * kMostThreads + 4 * t)) = f32x4{0.f, 0.f, 0.f, 0.f};
        } else {
#pragma unroll
            for (int j = 0; j < V; ++j) sums[u][j] = 0.f;
        }
    }
    // (sums that stand apart are a thread's own, and of a work-group that has one row at a time)
    auto apart = [&](int u, auto f) {
#pragma unroll
        for (int j = 0; j < V; j += 4) f(*reinterpret_cast<f32x4*>(shared + ((u * V + j) * kMostThreads + 4 * t)), j);
    };
    int round = 0;
    const int64_t step = (int64_t)gridDim.x * blockDim.y, begin = (int64_t)blockIdx.x * blockDim.y;
    auto row_at = [&](int64_t first) { return first + threadIdx.y < a.T ? first + threadIdx.y : a.T - 1; };      // (rows past the end repeat the last one and store nothing)
    Row<T, V, U, WHOLE> r, next;
    if (FEW && begin < a.T) next.load(a, rows::row_of<(U > 1)>(row_at(begin)), t, true);
    for (int64_t first = begin; first < a.T; first += step, round ^= 1) {
        const int64_t row = rows::row_of<(U > 1)>(row_at(first));
        const bool in = first + threadIdx.y < a.T;
        int t = threadIdx.x;
        if (FORMED) asm volatile("" : "+v"(t));  // (another number in each round, as far as the compiler knows: addresses are formed where they are used: kept ones spilled beside the rest)
        if (FEW) {
            r = next;
            if (first + step < a.T) next.load(a, rows::row_of<(U > 1)>(row_at(first + step)), t, true);
        } else {
            r.load(a, row, t, false);
        }
        const float rstd = r.rstd;
        Joined along{0.f, 0u};                   // sum of dhat x
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const Unit<V, WHOLE> unit(t + u * threads, C);
            float xv[V], dv[V], gamma[V], sum = 0.f;
            r.x[u].floats(xv);
            r.dy[u].floats(dv);
            if (!FEW) load_gamma(t, u);
            g[u].floats(gamma);
#pragma unroll
            for (int j = 0; j < V; ++j) {
                const float hat = xv[j] * rstd;
                if (WHOLE || unit.counts(j)) sum = fmaf(dv[j] * gamma[j], hat, sum);
                if (!APART && in) sums[u][j] = fmaf(dv[j], hat, sums[u][j]);
            }
            if (APART) {
                apart(u, [&](f32x4& s, int j) {
                    f32x4 v = s;
#pragma unroll
                    for (int e = 0; e < 4; ++e) v[e] = fmaf(dv[j + e], xv[j + e] * rstd, v[e]);
                    s = v;
                });
            }
            if (!WHOLE || unit.in()) along.sum += sum;
            unit_done<2 * U * V>();
        }
        if (!a.h) continue;
        along = join_row<true, false>(along, round);
        if (!in) continue;
        const float part = along.sum / (float)C;
#pragma unroll
        for (int u = 0; u < U; ++u) {
            r.x[u].keep_packed();
            r.dy[u].keep_packed();
            if (FEW) g[u].keep_packed();
        }
        if (FORMED) asm volatile("" : "+v"(t));
        by_streaming(a.streaming, [&](auto streaming) {
            constexpr bool S = decltype(streaming)::value;
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const Unit<V, WHOLE> unit(t + u * threads, C);
                if (!unit.in()) continue;
                float xv[V], dv[V], gamma[V], extra[V];
                r.x[u].floats(xv);
                r.dy[u].floats(dv);
                if (!FEW) load_gamma(t, u);
                g[u].floats(gamma);
                if (!FEW && a.dh) r.load_dh(a, row, t, u);
                if (a.dh) r.dh[u].floats(extra);
#pragma unroll
                for (int j = 0; j < V; ++j) {
                    dv[j] = rstd * fmaf(-xv[j] * rstd, part, dv[j] * gamma[j]);
                    if (a.dh) dv[j] += extra[j];
                }
                T* const to = at<T>(static_cast<T*>(a.h) + row * a.ldh, unit.start);
                // (FEW: what two units have both store, alike; dh was loaded in front of join_row, whose barrier, or a single wave's own order, has those loads ahead of every store here)
                if (FEW || WHOLE || unit.counted == 0) {
                    store<S>(to, dv);
                } else {                                             // (what another unit has too may be that one's result already, where dx is dh)
#pragma unroll
                    for (int j = 0; j < V; ++j)
                        if (unit.counts(j)) to[j] = from_float<T>(dv[j]);
                }
                unit_done<2 * U * V>();
            }
        });
    }
    if (!a.sums) return;
    // the rows of a work-group, then one line of the workspace
    float* const line = a.sums + (int64_t)blockIdx.x * C;
    if (APART || blockDim.y == 1) {
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const Unit<V, WHOLE> unit(t + u * threads, C);
            float v[V];
            if (APART) {
                apart(u, [&](const f32x4& s, int j) {
#pragma unroll
                    for (int e = 0; e < 4; ++e) v[j + e] = s[e];
                });
            } else {
#pragma unroll
                for (int j = 0; j < V; ++j) v[j] = sums[u][j];
            }
            if (WHOLE && unit.in()) store<false>(line + unit.start, v);
#pragma unroll
            for (int j = 0; j < V; ++j)
                if (!WHOLE && unit.counts(j)) line[unit.start + j] = v[j];
        }
        return;
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const Unit<V, WHOLE> unit(t + u * threads, C);
#pragma unroll
        for (int j = 0; j < V; ++j)
            if (unit.counts(j)) shared[threadIdx.y * C + unit.start + j] = sums[u][j];
    }
    __syncthreads();
    for (int c = threadIdx.y * threads + t; c < C; c += threads * (int)blockDim.y) {
        float sum = 0.f;
        for (int y = 0; y < (int)blockDim.y; ++y) sum += shared[y * C + c];
        line[c] = sum;
    }
}

// dgamma = the sum of `lines` lines of C floats: 32 columns of a work-group by 32 runs of lines, joined in LDS.
constexpr int kJoinColumns = 32, kJoinRuns = 32;
template <typename P>
__global__ __launch_bounds__(kJoinColumns* kJoinRuns) void join_kernel(const float* sums, int lines, int C, P* dgamma)
{
    __shared__ float parts[kJoinRuns][kJoinColumns];
    const int x = threadIdx.x % kJoinColumns, run = threadIdx.x / kJoinColumns, column = blockIdx.x * kJoinColumns + x;
    float sum = 0.f;
    if (column < C) {
#pragma unroll 8
        for (int i = run; i < lines; i += kJoinRuns) sum += sums[(int64_t)i * C + column];
    }
    parts[run][x] = sum;
    __syncthreads();
    if (run > 0 || column >= C) return;
    for (int i = 1; i < kJoinRuns; ++i) sum += parts[i][x];
    dgamma[column] = from_float<P>(sum);
}

}  // namespace rmsnorm
}  // namespace anr
