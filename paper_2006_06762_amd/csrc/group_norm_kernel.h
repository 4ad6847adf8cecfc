// Group norm with an activation, channels last, forward and backward.
//
// A group is Cg neighbouring channels of all pixels of an image: short runs of memory, C apart.  A work-group takes a
// chunk of whole groups (at least 128 bytes of a pixel's channels, so that lines are used whole) of a slab of pixels; its
// threads are columns of V channels by rows of pixels, and a thread keeps the sums of its V channels over its pixels.
//
// The statistics are sums in 64 bits, whose additions the vector units do at the rate of 32 bits: of the values (resident kernels, which then sum
// the squared differences from the mean), or, where x is read once for both, of each value's difference from one of the group's own, the
// first in the image, and of its square.  The mean square difference is then s2 / n - (s1 / n)^2, which loses the factor by which its
// second part exceeds it; that is (first - mean)^2 over the variance, at most n since the first value is one of the n: less than 2^-24 is lost
// below 2^28 values whatever they are.  (Means and squared differences in 32 bits, joined block by block, felt a first value that
// lies 1000 spreads out, 2e-5 of a spread in y, and grew with the number of joins.)  The mean is kept as two floats, its rounded value and the rest.
//
// Sums are joined by the threads of a work-group through LDS, those of slabs through the workspace, where the work-groups of the second
// kernel join them each for itself (fewer launches than a kernel that does), always in the same order.
//
// Where a work-group can hold a chunk of an image in its registers (resident kernels), it is read once, in one launch.
#pragma once
#include "anr_kernels.h"
#include "element_types.h"
#include "group_norm_plan.h"
#include "wave_join.h"

namespace anr {
namespace gnorm {

// Offsets of pixels; flat: one stride from pixel to pixel.
struct Pixels {
    int64_t sn, sh, sw;
    __device__ __forceinline__ int64_t at(int p, int W, const FastDiv& by_w, bool flat) const
    {
        if (flat) return (int64_t)p * sw;
        const int h = by_w.div(p);
        return (int64_t)h * sh + (int64_t)(p - h * W) * sw;
    }
};

struct Args {
    const void *x, *dy;
    void* y;
    const void *gamma, *beta;
    void *dgamma, *dbeta;
    float *mean, *rstd;
    double* stats;                  // forward: the two sums of each group over the slabs, [N][slabs][groups][2]
    double values;                  // of a group
    float* ws;                      // backward: the two sums of each group over the slabs, [N][slabs][groups][2]
    float* first;                   // forward: the value that each group's are relative to, [N][groups] (x may be overwritten in place)
    float* sums;                    // backward: sums of each channel over the slabs, [N][slabs][2][C]
    Pixels px, pdy, py;
    FastDiv by_w, by_cg;
    FastDiv by_each;                // resident: sums of a group in a row of threads, one a thread where its channels are of one group
    float eps;
    int N, HW, W, C, groups, cg, flat, param_dtype;
    int chunk;                      // channels of a chunk: whole groups
    int slabs, slab_pixels;
    bool halves;                    // resident: a chunk's pixel is half a line
    bool streaming;                 // y's stores go past L2: a chunk's pixel is whole lines of 128 bytes
};

// What a work-group works on.
struct Place {
    int slab, n, c0, channels, p0, p1;
    int columns, tx, ty, rows;      // of V channels; rows of threads
    __device__ __forceinline__ Place(const Args& a, int V, int threads = kThreads)
    {
        slab = blockIdx.x;
        n = blockIdx.z;
        int c = blockIdx.y;
        if (a.halves) {                 // of sixteen work-groups i and i + 8, which one XCD has, take neighbouring halves
            const int chunks = (int)gridDim.y, i = c + chunks * n, of16 = i & ~15;
            if (of16 + 16 <= chunks * a.N) {
                const int j = of16 + 2 * (i & 7) + ((i >> 3) & 1);
                n = j / chunks;
                c = j - n * chunks;
            }
        }
        c0 = c * a.chunk;
        channels = min(a.chunk, a.C - c0);
        p0 = slab * a.slab_pixels;
        p1 = min(a.HW, p0 + a.slab_pixels);
        columns = columns_of(channels, V);
        const int wide = min(columns, threads);
        rows = rows_of(channels, V, threads);
        ty = threadIdx.x / wide;
        tx = ty < rows ? threadIdx.x - ty * wide : columns;          // (threads that are left over have no column)
    }
};

// Parameter i of gamma or beta.
__device__ __forceinline__ float parameter(const void* p, int i, int dtype, float absent) { return p ? load_any(p, i, dtype) : absent; }

// The first value of each channel's group, for n of the chunk's channels from `first` on.
template <typename T>
__device__ __forceinline__ void origins(const Args& a, const T* x, int first, int n, float* out, int threads)
{
    for (int c = threadIdx.x; c < n; c += threads) out[c] = to_float(x[a.by_cg.div(first + c) * a.cg]);
}

// V values of a table of channels.
template <int V>
__device__ __forceinline__ void from_table(const float* table, int c, float (&out)[V])
{
    if constexpr (V % 4 == 0) {
#pragma unroll
        for (int i = 0; i < V; i += 4) {
            const f32x4 v = *reinterpret_cast<const f32x4*>(table + c + i);
#pragma unroll
            for (int j = 0; j < 4; ++j) out[i + j] = v[j];
        }
    } else {
#pragma unroll
        for (int i = 0; i < V; ++i) out[i] = table[c + i];
    }
}

// A mean as its rounded value and the rest.
__device__ __forceinline__ void two_floats(double mean, float& high, float& low)
{
    high = (float)mean;
    low = (float)(mean - (double)high);
}

// First kernel of the forward pass: the two sums of each group of the chunk over the slab.
template <typename T, int V>
__global__ __launch_bounds__(kThreads) void stats_kernel(const Args a)
{
    extern __shared__ __attribute__((aligned(16))) float shared[];   // the table, then the sums, [2][V][rows][columns] in 64 bits
    const Place s(a, V);
    const int table = table_floats(table_channels(s.channels, V)), all = s.rows * s.channels;
    double* const lds = reinterpret_cast<double*>(shared + table);
    const T* const x = static_cast<const T*>(a.x) + s.n * a.px.sn + s.c0;
    for (int base = 0; base < s.columns; base += kThreads) {         // (one round but for groups of thousands of channels)
        const int here = min(s.channels - base * V, kThreads * V), col = base + s.tx;
        __syncthreads();
        origins(a, x, base * V, here, shared, kThreads);
        __syncthreads();
        if (col >= s.columns) continue;
        double sum[V], squares[V];
        float origin[V];
#pragma unroll
        for (int i = 0; i < V; ++i) sum[i] = squares[i] = 0.;
        from_table<V>(shared, s.tx * V, origin);
        const T* const xc = x + col * V;
#pragma unroll 4
        for (int p = s.p0 + s.ty; p < s.p1; p += s.rows) {
            float v[V];
            load_floats<T, V>(xc + a.px.at(p, a.W, a.by_w, a.flat), v);
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const double d = (double)v[i] - (double)origin[i];
                sum[i] += d;
                squares[i] = fma(d, d, squares[i]);
            }
        }
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const int at = (i * s.rows + s.ty) * s.columns + col;
            lds[at] = sum[i];
            lds[all + at] = squares[i];
        }
    }
    __syncthreads();
    const int groups = s.channels / a.cg, wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    for (int g = wave; g < groups; g += kThreads / 64) {
        double sum = 0., squares = 0.;
        for (int e = lane; e < s.rows * a.cg; e += 64) {
            const int row = a.by_cg.div(e), c = g * a.cg + e - row * a.cg, at = (c % V * s.rows + row) * s.columns + c / V;
            sum += lds[at];
            squares += lds[all + at];
        }
        sum = wave_sum(sum);
        squares = wave_sum(squares);
        if (lane == 0) {
            double* const at = a.stats + 2 * (((int64_t)s.n * a.slabs + s.slab) * a.groups + s.c0 / a.cg + g);
            at[0] = sum;
            at[1] = squares;
            if (s.slab == 0) a.first[(int64_t)s.n * a.groups + s.c0 / a.cg + g] = to_float(x[g * a.cg]);
        }
    }
}

// Second kernel of the forward pass.
template <typename T, int V, int ACT>
__global__ __launch_bounds__(kThreads) void apply_kernel(const Args a)
{
    constexpr bool QUICK = sizeof(T) == 2;
    extern __shared__ __attribute__((aligned(16))) float shared[];   // tables of mean, scale and shift, then [groups] of (mean, rest of the mean, rstd)
    const Place s(a, V);
    const int table = table_floats(table_channels(s.channels, V));
    float* const lds = shared + 3 * table;
    const int groups = s.channels / a.cg, wave = threadIdx.x >> 6, lane = threadIdx.x & 63, g0 = s.c0 / a.cg;
    for (int g = wave; g < groups; g += kThreads / 64) {
        const double* const at = a.stats + 2 * ((int64_t)s.n * a.slabs * a.groups + g0 + g);
        double sum = 0., squares = 0.;
        for (int i = lane; i < a.slabs; i += 64) {
            sum += at[2 * (int64_t)i * a.groups];
            squares += at[2 * (int64_t)i * a.groups + 1];
        }
        const double mean = wave_sum(sum) / a.values, var = wave_sum(squares) / a.values - mean * mean;    // (the mean relative to the first value)
        const float rstd = 1.f / sqrtf((float)((var < 0. ? 0. : var) + (double)a.eps));
        if (lane == 0) {
            float high, low;
            two_floats(mean + (double)a.first[(int64_t)s.n * a.groups + g0 + g], high, low);
            lds[3 * g] = high;
            lds[3 * g + 1] = low;
            lds[3 * g + 2] = rstd;
            if (s.slab == 0 && a.mean) a.mean[(int64_t)s.n * a.groups + g0 + g] = high;
            if (s.slab == 0 && a.rstd) a.rstd[(int64_t)s.n * a.groups + g0 + g] = rstd;
        }
    }
    const T* const x = static_cast<const T*>(a.x) + s.n * a.px.sn + s.c0;
    T* const y = static_cast<T*>(a.y) + s.n * a.py.sn + s.c0;
    for (int base = 0; base < s.columns; base += kThreads) {
        const int first = base * V, here = min(s.channels - first, kThreads * V), col = base + s.tx;
        __syncthreads();
        for (int c = threadIdx.x; c < here; c += kThreads) {
            const int g = a.by_cg.div(first + c);
            const float scale = lds[3 * g + 2] * parameter(a.gamma, s.c0 + first + c, a.param_dtype, 1.f);
            shared[c] = lds[3 * g];
            shared[table + c] = scale;
            shared[2 * table + c] = fmaf(-lds[3 * g + 1], scale, parameter(a.beta, s.c0 + first + c, a.param_dtype, 0.f));
        }
        __syncthreads();
        if (col >= s.columns) continue;
        float mean[V], scale[V], shift[V];
        from_table<V>(shared, s.tx * V, mean);
        from_table<V>(shared + table, s.tx * V, scale);
        from_table<V>(shared + 2 * table, s.tx * V, shift);
        by_streaming(a.streaming, [&](auto streaming) {
#pragma unroll 4
            for (int p = s.p0 + s.ty; p < s.p1; p += s.rows) {
                float v[V];
                load_floats<T, V>(x + a.px.at(p, a.W, a.by_w, a.flat) + col * V, v);
#pragma unroll
                for (int i = 0; i < V; ++i) v[i] = activation<ACT, QUICK>(fmaf(v[i] - mean[i], scale[i], shift[i]));
                store_pack<decltype(streaming)::value>(y + a.py.at(p, a.W, a.by_w, a.flat) + col * V, pack_floats<T, V>(v));
            }
        });
    }
}

// What the backward pass needs of each channel: tables of mean, rstd, gamma and beta, for n of the chunk's channels from `first` on.
__device__ __forceinline__ void channel_tables(const Args& a, const Place& s, int first, int n, float* out, int table, int threads)
{
    for (int c = threadIdx.x; c < n; c += threads) {
        const int64_t g = (int64_t)s.n * a.groups + s.c0 / a.cg + a.by_cg.div(first + c);
        out[c] = a.mean[g];
        out[table + c] = a.rstd[g];
        out[2 * table + c] = parameter(a.gamma, s.c0 + first + c, a.param_dtype, 1.f);
        out[3 * table + c] = parameter(a.beta, s.c0 + first + c, a.param_dtype, 0.f);
    }
}
template <int V>
struct Channels {
    float mean[V], rstd[V], gamma[V], beta[V];
    __device__ __forceinline__ void load(const float* tables, int table, int c)
    {
        from_table<V>(tables, c, mean);
        from_table<V>(tables + table, c, rstd);
        from_table<V>(tables + 2 * table, c, gamma);
        from_table<V>(tables + 3 * table, c, beta);
    }
    // xhat and dz of one element
    template <int ACT, bool QUICK>
    __device__ __forceinline__ void element(int i, float x, float dy, float& hat, float& dz) const
    {
        hat = (x - mean[i]) * rstd[i];
        float slope = 1.f;
        if (ACT != ANR_ACT_NONE) activation_and_slope<ACT, QUICK>(fmaf(hat, gamma[i], beta[i]), slope);
        dz = dy * slope;
    }
};

// First kernel of the backward pass: sums of dz and dz xhat over the slab, of each channel and, with gamma, of each group.  A thread adds 32 pixels in
// 32 bits and those sums in 64, in its place in LDS: one after another in 32 bits, 1500 pixels of one value were 250 units of the last
// place off, and the number of pixels has no bound.
template <typename T, int V, int ACT>
__global__ __launch_bounds__(kThreads) void backward_sums_kernel(const Args a)
{
    constexpr bool QUICK = sizeof(T) == 2;
    extern __shared__ __attribute__((aligned(16))) float shared[];   // the tables, then the sums, [2][V][rows][columns] in 64 bits
    const Place s(a, V);
    const int table = table_floats(table_channels(s.channels, V)), all = s.rows * s.channels;
    double* const lds = reinterpret_cast<double*>(shared + 4 * table);
    const T* const x = static_cast<const T*>(a.x) + s.n * a.px.sn + s.c0;
    const T* const dy = static_cast<const T*>(a.dy) + s.n * a.pdy.sn + s.c0;
    for (int base = 0; base < s.columns; base += kThreads) {
        const int col = base + s.tx;
        __syncthreads();
        channel_tables(a, s, base * V, min(s.channels - base * V, kThreads * V), shared, table, kThreads);
        __syncthreads();
        if (col >= s.columns) continue;
        Channels<V> ch;
        ch.load(shared, table, s.tx * V);
        int p = s.p0 + s.ty;
        auto add = [&](auto first) {
            float sum[V], with_hat[V];
#pragma unroll
            for (int i = 0; i < V; ++i) sum[i] = with_hat[i] = 0.f;
            const int end = min(s.p1, p + 32 * s.rows);
#pragma unroll 4
            for (; p < end; p += s.rows) {
                float v[V], d[V];
                load_floats<T, V>(x + a.px.at(p, a.W, a.by_w, a.flat) + col * V, v);
                load_floats<T, V>(dy + a.pdy.at(p, a.W, a.by_w, a.flat) + col * V, d);
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    float hat, dz;
                    ch.template element<ACT, QUICK>(i, v[i], d[i], hat, dz);
                    sum[i] += dz;
                    with_hat[i] = fmaf(dz, hat, with_hat[i]);
                }
            }
#pragma unroll
            for (int i = 0; i < V; ++i) {
                double* const at = lds + (i * s.rows + s.ty) * s.columns + col;
                at[0] = (double)sum[i] + (decltype(first)::value ? 0. : at[0]);
                at[all] = (double)with_hat[i] + (decltype(first)::value ? 0. : at[all]);
            }
        };
        add(std::true_type{});
        while (p < s.p1) add(std::false_type{});
    }
    __syncthreads();
    float* const out = a.sums + ((int64_t)s.n * a.slabs + s.slab) * 2 * a.C + s.c0;
    auto first_row = [&](int which, int c) { return which * all + c % V * s.rows * s.columns + c / V; };
    for (int e = threadIdx.x; e < 2 * s.channels; e += kThreads) {   // neighbouring threads take neighbouring columns
        const int which = e >= s.channels, i = (e - which * s.channels) / s.columns, col = e - which * s.channels - i * s.columns, c = col * V + i;
        double* const at = lds + which * all + i * s.rows * s.columns + col;
        double sum = 0.;
#pragma unroll 8
        for (int r = 0; r < s.rows; ++r) sum += at[r * s.columns];
        out[(int64_t)which * a.C + c] = (float)sum;
        at[0] = sum * (double)parameter(a.gamma, s.c0 + c, a.param_dtype, 1.f);      // (row 0, which this thread alone reads)
    }
    __syncthreads();
    float* const of_groups = a.ws + 2 * (((int64_t)s.n * a.slabs + s.slab) * a.groups + s.c0 / a.cg);
    for (int e = threadIdx.x; e < 2 * (s.channels / a.cg); e += kThreads) {
        double sum = 0.;
#pragma unroll 8
        for (int c = (e >> 1) * a.cg; c < ((e >> 1) + 1) * a.cg; ++c) sum += lds[first_row(e & 1, c)];
        of_groups[e] = (float)sum;
    }
}

// dgamma and dbeta of the chunk: sums over the images' slabs, which the threads of a channel share, in 64 bits (there are as many as images).
__device__ __forceinline__ void parameter_gradients(const Args& a, double* lds, int threads)
{
    const int c0 = blockIdx.y * a.chunk, channels = min(a.chunk, a.C - c0), sums = 2 * channels;
    const int64_t parts = (int64_t)a.N * a.slabs;
    for (int base = 0; base < sums; base += threads) {
        const int here = min(sums - base, threads), shares = threads / here, share = threadIdx.x / here, e = base + threadIdx.x - share * here;
        const int which = e >= channels, c = c0 + e - which * channels;
        double sum = 0.;
        if (share < shares) {
#pragma unroll 8
            for (int64_t i = share; i < parts; i += shares) sum += (double)a.sums[(i * 2 + which) * a.C + c];
        }
        __syncthreads();
        lds[threadIdx.x] = sum;
        __syncthreads();
        void* const out = which ? a.dgamma : a.dbeta;
        if (share > 0 || !out) continue;
        for (int i = 1; i < shares; ++i) sum += lds[i * here + threadIdx.x];
        store_any(out, c, a.param_dtype, (float)sum);
    }
}

__global__ __launch_bounds__(kThreads) void backward_parameters_kernel(const Args a)
{
    __shared__ double lds[kThreads];
    parameter_gradients(a, lds, kThreads);
}

// Second kernel: dx, and in work-groups of their own, behind the last image's, the parameters' gradients (behind the slabs, where they moved the others to
// other XCDs than those whose L2 has what the first kernel read there, 2 x 96^2 x 320 in float32 took 32 us, so 27).
template <typename T, int V, int ACT>
__global__ __launch_bounds__(kThreads) void backward_apply_kernel(const Args a)
{
    constexpr bool QUICK = sizeof(T) == 2;
    extern __shared__ __attribute__((aligned(16))) float shared[];   // the tables, those of the group's two means, and [groups] of the means
    if ((int)blockIdx.z == a.N) {
        if (blockIdx.x == 0) parameter_gradients(a, reinterpret_cast<double*>(shared), kThreads);
        return;
    }
    const Place s(a, V);
    const int table = table_floats(table_channels(s.channels, V));
    float* const means = shared + 6 * table;
    for (int g = threadIdx.x >> 6; g < s.channels / a.cg; g += kThreads / 64) {
        const float* const at = a.ws + 2 * ((int64_t)s.n * a.slabs * a.groups + s.c0 / a.cg + g);
        float dz = 0.f, with_hat = 0.f;
        for (int i = threadIdx.x & 63; i < a.slabs; i += 64) {
            dz += at[2 * (int64_t)i * a.groups];
            with_hat += at[2 * (int64_t)i * a.groups + 1];
        }
        dz = wave_sum(dz);
        with_hat = wave_sum(with_hat);
        if ((threadIdx.x & 63) == 0) {
            means[2 * g] = dz / (float)a.values;
            means[2 * g + 1] = with_hat / (float)a.values;
        }
    }
    const T* const x = static_cast<const T*>(a.x) + s.n * a.px.sn + s.c0;
    const T* const dy = static_cast<const T*>(a.dy) + s.n * a.pdy.sn + s.c0;
    T* const dx = static_cast<T*>(a.y) + s.n * a.py.sn + s.c0;
    for (int base = 0; base < s.columns; base += kThreads) {
        const int first = base * V, here = min(s.channels - first, kThreads * V), col = base + s.tx;
        __syncthreads();
        channel_tables(a, s, first, here, shared, table, kThreads);
        for (int c = threadIdx.x; c < here; c += kThreads) {
            const int g = a.by_cg.div(first + c);
            shared[4 * table + c] = means[2 * g];
            shared[5 * table + c] = means[2 * g + 1];
        }
        __syncthreads();
        if (col >= s.columns) continue;
        Channels<V> ch;
        ch.load(shared, table, s.tx * V);
        float mean_dz[V], mean_with_hat[V];
        from_table<V>(shared + 4 * table, s.tx * V, mean_dz);
        from_table<V>(shared + 5 * table, s.tx * V, mean_with_hat);
        by_streaming(a.streaming, [&](auto streaming) {
#pragma unroll 2
            for (int p = s.p0 + s.ty; p < s.p1; p += s.rows) {
                float v[V], d[V];
                load_floats<T, V>(x + a.px.at(p, a.W, a.by_w, a.flat) + col * V, v);
                load_floats<T, V>(dy + a.pdy.at(p, a.W, a.by_w, a.flat) + col * V, d);
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    float hat, dz;
                    ch.template element<ACT, QUICK>(i, v[i], d[i], hat, dz);
                    v[i] = ch.rstd[i] * (fmaf(dz, ch.gamma[i], -mean_dz[i]) - hat * mean_with_hat[i]);
                }
                store_pack<decltype(streaming)::value>(dx + a.py.at(p, a.W, a.by_w, a.flat) + col * V, pack_floats<T, V>(v));
            }
        });
    }
}

// ---- resident: a work-group holds its chunk of an image, at most R vectors of kHeldChannels channels a thread

// Means over the work-group's rows and each group's channels of what a thread has summed of each channel; that of group g at
// result[g].  (By a division: that of equal values is that value.)  `part`: [rows][channels], or a place a thread where its channels are of one group.
template <typename S, int V>
__device__ __forceinline__ void group_means_of(const Args& a, const Place& s, const S (&v)[V], S* part, S* result, int threads)
{
    const bool whole = a.cg % V == 0;
    const int width = whole ? s.columns : s.channels, each = whole ? a.cg / V : a.cg;       // of a row, of a group in it
    if (s.tx < s.columns) {
        if (whole) {
            S sum = v[0];
#pragma unroll
            for (int i = 1; i < V; ++i) sum += v[i];
            part[s.ty * width + s.tx] = sum;
        } else {
#pragma unroll
            for (int i = 0; i < V; ++i) part[s.ty * width + s.tx * V + i] = v[i];
        }
    }
    __syncthreads();
    const int groups = s.channels / a.cg, lane = threadIdx.x & 63, entries = s.rows * each;
    for (int g = threadIdx.x >> 6; g < groups; g += threads >> 6) {
        S sum = 0;
        for (int e = lane; e < entries; e += 64) {
            const int row = a.by_each.div(e);
            sum += part[row * width + g * each + e - row * each];
        }
        sum = wave_sum(sum);
        if (lane == 0) result[g] = sum / (S)a.values;
    }
    __syncthreads();
}

template <typename T, int ACT, int R>
__global__ __launch_bounds__(1024) void resident_kernel(const Args a)
{
    constexpr bool QUICK = sizeof(T) == 2;
    constexpr int V = kHeldChannels;
    extern __shared__ __attribute__((aligned(16))) float shared[];   // tables of scale and shift, then [groups] and [rows][channels] in 64 bits
    const int threads = blockDim.x;
    const Place s(a, V, threads);
    const int table = table_floats(s.channels), groups = s.channels / a.cg;
    double *const result = reinterpret_cast<double*>(shared + 2 * table), *const part = result + table_floats(groups);
    float *const result32 = reinterpret_cast<float*>(result), *const part32 = reinterpret_cast<float*>(part);
    const T* const x = static_cast<const T*>(a.x) + s.n * a.px.sn + s.c0;
    const int col = min(s.tx, s.columns - 1) * V, mine = s.tx < s.columns && s.ty < a.HW ? (a.HW - s.ty + s.rows - 1) / s.rows : 0;
    using Raw = Pack<T, V>;
    Raw raw[R];
#pragma unroll
    for (int r = 0; r < R; ++r) raw[r] = *reinterpret_cast<const Raw*>(x + a.px.at(min(s.ty + r * s.rows, a.HW - 1), a.W, a.by_w, a.flat) + col);
    for (int c = threadIdx.x; c < s.channels; c += threads) {
        shared[c] = parameter(a.gamma, s.c0 + c, a.param_dtype, 1.f);
        shared[table + c] = parameter(a.beta, s.c0 + c, a.param_dtype, 0.f);
    }
    double total[V];
#pragma unroll
    for (int i = 0; i < V; ++i) total[i] = 0.;
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
        for (int i = 0; i < V; ++i) total[i] += (double)(r < mine ? to_float(raw[r].v[i]) : 0.f);
    if constexpr (QUICK && R == 16) {                                 // (what is held are the 16 bits: the floats, kept from sum to sum, do not fit the registers)
        typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
#pragma unroll
        for (int r = 0; r < R; ++r) {
            u32x2 bits = __builtin_bit_cast(u32x2, raw[r]);
            asm("" : "+v"(bits));
            raw[r] = __builtin_bit_cast(Raw, bits);
        }
    }
    group_means_of<double, V>(a, s, total, part, result, threads);
    float high[V], low[V], sum[V];                                   // the mean, and its rest
#pragma unroll
    for (int i = 0; i < V; ++i) {
        two_floats(result[a.by_cg.div(col + i)], high[i], low[i]);
        sum[i] = 0.f;
    }
    const float own_mean = threadIdx.x < groups ? (float)result[threadIdx.x] : 0.f;
    __syncthreads();
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const float d = to_float(raw[r].v[i]) - high[i] - low[i];
            sum[i] = r < mine ? fmaf(d, d, sum[i]) : sum[i];
        }
    group_means_of<float, V>(a, s, sum, part32, result32, threads);
    if (threadIdx.x < groups) {
        const int64_t g = (int64_t)s.n * a.groups + s.c0 / a.cg + threadIdx.x;
        if (a.mean) a.mean[g] = own_mean;
        if (a.rstd) a.rstd[g] = 1.f / sqrtf(result32[threadIdx.x] + a.eps);
    }
    float scale[V], shift[V];
    from_table<V>(shared, col, scale);
    from_table<V>(shared + table, col, shift);
#pragma unroll
    for (int i = 0; i < V; ++i) {
        scale[i] *= 1.f / sqrtf(result32[a.by_cg.div(col + i)] + a.eps);
        shift[i] = fmaf(-low[i], scale[i], shift[i]);
    }
    T* const y = static_cast<T*>(a.y) + s.n * a.py.sn + s.c0;
#pragma unroll
    for (int r = 0; r < R; ++r) {
        if (r >= mine) continue;
        float v[V];
#pragma unroll
        for (int i = 0; i < V; ++i) v[i] = activation<ACT, QUICK>(fmaf(to_float(raw[r].v[i]) - high[i], scale[i], shift[i]));
        store_floats<T, V>(y + a.py.at(s.ty + r * s.rows, a.W, a.by_w, a.flat) + col, v);
    }
}

// Backward, resident: writes the sums of each channel over the image, which the kernel of the parameters' gradients takes, and dx.
template <typename T, int ACT, int R>
__global__ __launch_bounds__(1024) void backward_resident_kernel(const Args a)
{
    constexpr bool QUICK = sizeof(T) == 2;
    constexpr int V = kHeldChannels;
    extern __shared__ __attribute__((aligned(16))) float shared[];   // the tables, [2][channels], [groups] of two means, [rows][2][channels], [threads] in 64 bits
    const int threads = blockDim.x;
    const Place s(a, V, threads);
    const int table = table_floats(s.channels), groups = s.channels / a.cg;
    float *const total = shared + 4 * table, *const means = total + 2 * table, *const part = means + table_floats(2 * groups);
    const T* const x = static_cast<const T*>(a.x) + s.n * a.px.sn + s.c0;
    const T* const dy = static_cast<const T*>(a.dy) + s.n * a.pdy.sn + s.c0;
    const int col = min(s.tx, s.columns - 1) * V, mine = s.tx < s.columns && s.ty < a.HW ? (a.HW - s.ty + s.rows - 1) / s.rows : 0;
    Pack<T, V> rx[R], rd[R];
#pragma unroll
    for (int r = 0; r < R; ++r) {
        const int p = min(s.ty + r * s.rows, a.HW - 1);
        rx[r] = *reinterpret_cast<const Pack<T, V>*>(x + a.px.at(p, a.W, a.by_w, a.flat) + col);
        rd[r] = *reinterpret_cast<const Pack<T, V>*>(dy + a.pdy.at(p, a.W, a.by_w, a.flat) + col);
    }
    channel_tables(a, s, 0, s.channels, shared, table, threads);
    __syncthreads();
    Channels<V> ch;
    ch.load(shared, table, col);
    float sum[V], with_hat[V];
#pragma unroll
    for (int i = 0; i < V; ++i) sum[i] = with_hat[i] = 0.f;
#pragma unroll
    for (int r = 0; r < R; ++r) {
        if (r >= mine) continue;
#pragma unroll
        for (int i = 0; i < V; ++i) {
            float hat, dz;
            ch.template element<ACT, QUICK>(i, to_float(rx[r].v[i]), to_float(rd[r].v[i]), hat, dz);
            sum[i] += dz;
            with_hat[i] = fmaf(dz, hat, with_hat[i]);
            if (!QUICK) {                                             // (float32: what is held from here on)
                rx[r].v[i] = from_float<T>(hat);
                rd[r].v[i] = from_float<T>(dz);
            }
        }
    }
    if (s.tx < s.columns) {
#pragma unroll
        for (int i = 0; i < V; ++i) {
            part[(2 * s.ty) * s.channels + col + i] = sum[i];
            part[(2 * s.ty + 1) * s.channels + col + i] = with_hat[i];
        }
    }
    __syncthreads();
    // the threads of a channel share the rows
    double* const shares_of = reinterpret_cast<double*>(part + 2 * s.rows * s.channels);
    for (int base = 0; base < 2 * s.channels; base += threads) {
        const int here = min(2 * s.channels - base, threads), shares = threads / here, share = threadIdx.x / here, e = base + threadIdx.x - share * here;
        const int which = e >= s.channels, c = e - which * s.channels;
        double v = 0.;
        if (share < shares) {
#pragma unroll 4
            for (int r = share; r < s.rows; r += shares) v += (double)part[(2 * r + which) * s.channels + c];
        }
        __syncthreads();
        shares_of[threadIdx.x] = v;
        __syncthreads();
        if (share > 0) continue;
        for (int i = 1; i < shares; ++i) v += shares_of[i * here + threadIdx.x];
        a.sums[((int64_t)s.n * 2 + which) * a.C + s.c0 + c] = (float)v;
        total[which * table + c] = (float)v * shared[2 * table + c];
    }
    if (!a.y) return;
    __syncthreads();
    for (int e = threadIdx.x; e < 2 * groups; e += threads) {
        double v = 0.;
        for (int c = 0; c < a.cg; ++c) v += (double)total[(e & 1) * table + (e >> 1) * a.cg + c];
        means[e] = (float)(v / a.values);
    }
    __syncthreads();
    float mean_dz[V], mean_with_hat[V];
#pragma unroll
    for (int i = 0; i < V; ++i) {
        const int g = a.by_cg.div(col + i);
        mean_dz[i] = means[2 * g];
        mean_with_hat[i] = means[2 * g + 1];
    }
    T* const dx = static_cast<T*>(a.y) + s.n * a.py.sn + s.c0;
#pragma unroll
    for (int r = 0; r < R; ++r) {
        if (r >= mine) continue;
        float v[V];
#pragma unroll
        for (int i = 0; i < V; ++i) {
            float hat = to_float(rx[r].v[i]), dz = to_float(rd[r].v[i]);
            if (QUICK) ch.template element<ACT, QUICK>(i, hat, dz, hat, dz);
            v[i] = ch.rstd[i] * (fmaf(dz, ch.gamma[i], -mean_dz[i]) - hat * mean_with_hat[i]);
        }
        store_floats<T, V>(dx + a.py.at(s.ty + r * s.rows, a.W, a.by_w, a.flat) + col, v);
    }
}

// Nothing to norm: means of zero, spreads of zero, gradients of zero.
__global__ __launch_bounds__(kThreads) void empty_kernel(const Args a, bool backward)
{
    const int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x;
    if (!backward && i < (int64_t)a.N * a.groups) {
        if (a.mean) a.mean[i] = 0.f;
        if (a.rstd) a.rstd[i] = 1.f / sqrtf(a.eps);
    }
    if (backward && i < a.C) {
        if (a.dgamma) store_any(a.dgamma, i, a.param_dtype, 0.f);
        if (a.dbeta) store_any(a.dbeta, i, a.param_dtype, 0.f);
    }
}

}  // namespace gnorm
}  // namespace anr
