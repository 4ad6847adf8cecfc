// Gated feed-forward block: which kernels a call runs, and the kernels between its products.
//
//   few tokens     ff_rows_kernel.h: two launches, each reads its weights once
//   16-bit types   mm16_kernel.h: gate, up, activation and product in one launch, then the down projection; backward
//                  three (dh with dg, du and h where they are formed; dx; the weights' gradients together)
//   float32        the library's GEMM (gemm.hip): gate, up, activation and product in one launch of its form for two matrices, the other
//                  products with the kernels here around them
#include <algorithm>

#include "blocks_internal.h"
#include "element_types.h"
#include "ff_rows_kernel.h"
#include "gemm_split_plan.h"
#include "mm16_launch.h"

namespace anr {
namespace {

constexpr int kThreads = 256;
// Calls of few tokens (ff_rows_kernel.h): sixteen, in float32 32, and up to 64 while each work-group's pass over them costs less than the tiles of 128 tokens that
// are mostly empty. us, T tokens so / in tiles: 16 bits, 1024 -> 2816 T = 17 15.4 / 21.6, 48 21.9 / 22.8, 64 23.9 / 23.6, 1536 -> 4096 33 24.7 / 26.4, 40 26.5 /
// 26.5, 48 28.2 / 27.0, 2048 -> 5632 17 29.3 / 29.5, 20 30.7 / 29.0, 64 51.7 / 32.5, 2560 -> 6912 17 40.1 / 41.3, 20 42.7 / 41.6, 4096 -> 11264 17 73.7 / 67.4, 64
// 140 / 73; float32, 1024 -> 2816 17 24 / 40, 48 38 / 41, 64 43.5 / 41.3, 1536 -> 4096 32 38 / 51, 48 51.8 / 51.3, 2048 -> 5632 17 60 / 69, 32 75.8 / 73.0, 64
// 116 / 75, 2560 -> 6912 32 97 / 88, 4096 -> 11264 17 144 / 210, 32 185 / 215, 48 246 / 217.
bool few_tokens(const anr_gated_ff_desc& d)
{
    const bool f32 = d.dtype == ANR_F32;
    return d.T <= (f32 ? 32 : 16) || (d.T <= 64 && d.T * d.C * d.F <= (int64_t)(f32 ? 150000000 : 220000000));
}

size_t whole_lines(size_t bytes) { return (bytes + 255) & ~(size_t)255; }

// ---- float32: the kernels between the products

// h = act(gate) up, all [T,F]; h packed.
template <int ACT>
__global__ __launch_bounds__(kThreads) void product_of_gate_kernel(const float* gate, const float* up, int64_t ld, float* h, int64_t T, int64_t F)
{
    for (int64_t t = blockIdx.y; t < T; t += gridDim.y)
        for (int64_t f = (int64_t)blockIdx.x * kThreads + threadIdx.x; f < F; f += (int64_t)gridDim.x * kThreads)
            h[t * F + f] = activation<ACT, false>(gate[t * ld + f]) * up[t * ld + f];
}

// From dh, gate and up [T,F]: dgu [T, 2F] (dg and du side by side), the same turned [2F, T], and h [T,F].
template <int ACT>
__global__ __launch_bounds__(kThreads) void hidden_gradients_kernel(const float* dh, const float* gate, const float* up, int64_t ld, float* dgu, float* turned, float* h,
                                                                    int64_t T, int64_t F)
{
    __shared__ float tile[2][32][33];
    const int x = threadIdx.x & 31, y = threadIdx.x >> 5;
    const int64_t f0 = (int64_t)blockIdx.x * 32;
    for (int64_t t0 = (int64_t)blockIdx.y * 32; t0 < T; t0 += (int64_t)gridDim.y * 32) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int64_t t = t0 + y + 8 * i, f = f0 + x;
            if (t >= T || f >= F) continue;
            const float g = gate[t * ld + f], u = up[t * ld + f], d = dh[t * F + f];
            float slope;
            const float a = activation_and_slope<ACT, false>(g, slope);
            const float dg = d * u * slope, du = d * a;
            dgu[t * 2 * F + f] = dg;
            dgu[t * 2 * F + F + f] = du;
            h[t * F + f] = a * u;
            tile[0][y + 8 * i][x] = dg;
            tile[1][y + 8 * i][x] = du;
        }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int64_t f = f0 + y + 8 * i, t = t0 + x;
            if (f >= F || t >= T) continue;
            turned[f * T + t] = tile[0][x][y + 8 * i];
            turned[(F + f) * T + t] = tile[1][x][y + 8 * i];
        }
        __syncthreads();
    }
}

// What a matrix [R,C] is laid out as: packed, or turned, [C,R].
struct Layout {
    const float* in;
    int64_t ld, R, C;
    float* out;
    bool turned;
};
struct Layouts {
    Layout l[3];
};
__global__ __launch_bounds__(kThreads) void lay_out_kernel(const Layouts all)
{
    __shared__ float tile[32][33];
    const Layout& l = all.l[blockIdx.z];
    const int x = threadIdx.x & 31, y = threadIdx.x >> 5;
    const int64_t c0 = (int64_t)blockIdx.x * 32;
    if (c0 >= l.C) return;
    for (int64_t r0 = (int64_t)blockIdx.y * 32; r0 < l.R; r0 += (int64_t)gridDim.y * 32) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int64_t r = r0 + y + 8 * i, c = c0 + x;
            if (r >= l.R || c >= l.C) continue;
            if (l.turned) tile[y + 8 * i][x] = l.in[r * l.ld + c];
            else l.out[r * l.C + c] = l.in[r * l.ld + c];
        }
        if (!l.turned) continue;
        __syncthreads();
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (c0 + y + 8 * i < l.C && r0 + x < l.R) l.out[(c0 + y + 8 * i) * l.R + r0 + x] = tile[x][y + 8 * i];
        __syncthreads();
    }
}

// D [M,N] in T = the sum of the `splits` packed matrices at `parts`, in their order; `units` of V columns a row.
template <typename T, int V>
__global__ __launch_bounds__(kThreads) void join_kernel(const float* parts, int splits, T* d, int64_t ldd, int64_t M, int64_t units)
{
    const int64_t each = M * units, i = (int64_t)blockIdx.x * kThreads + threadIdx.x;
    if (i >= each) return;
    const int64_t m = each < (int64_t)1 << 31 ? (int64_t)((uint32_t)i / (uint32_t)units) : i / units;
    float sum[V];
    load_floats<float, V>(parts + i * V, sum);
#pragma unroll 4
    for (int s = 1; s < splits; ++s) {
        float v[V];
        load_floats<float, V>(parts + (s * each + i) * V, v);
#pragma unroll
        for (int e = 0; e < V; ++e) sum[e] += v[e];
    }
    store_floats<T, V>(d + m * ldd + (i - m * units) * V, sum);
}

template <typename T>
__global__ __launch_bounds__(kThreads) void zero_kernel(T* d, int64_t ldd, int64_t M, int64_t N)
{
    for (int64_t m = blockIdx.y; m < M; m += gridDim.y)
        for (int64_t n = (int64_t)blockIdx.x * kThreads + threadIdx.x; n < N; n += (int64_t)gridDim.x * kThreads) d[m * ldd + n] = T(0.f);
}

template <typename T>
hipError_t launch_join(const float* parts, int splits, T* d, int64_t ldd, int64_t M, int64_t N, hipStream_t stream)
{
    auto with = [&](auto v) {
        constexpr int V = decltype(v)::value;
        const int64_t groups = (M * (N / V) + kThreads - 1) / kThreads;
        return launch_kernel(join_kernel<T, V>, dim3((unsigned)groups), dim3(kThreads), 0, stream, parts, splits, d, ldd, M, N / V);
    };
    // 16-byte loads: two parts of 2048 x 768 took 7.4 us with loads of single floats, 5.0 so
    if (N % 4 == 0 && ldd % 4 == 0 && reinterpret_cast<uintptr_t>(d) % (4 * sizeof(T)) == 0) return with(std::integral_constant<int, 4>{});
    return with(std::integral_constant<int, 1>{});
}

dim3 grid_of(int64_t columns, int64_t per, int64_t rows, int64_t rows_per)
{
    return dim3((unsigned)((columns + per - 1) / per), (unsigned)std::max<int64_t>(1, std::min<int64_t>((rows + rows_per - 1) / rows_per, 65535)));
}

// C [M,N] = A [M,K] B, B as [N,K] (nk) or [K,N]; `batch` of them with these steps.
hipError_t gemm(const float* A, int64_t lda, const float* B, int64_t ldb, bool nk, float* C, int64_t ldc, int64_t M, int64_t N, int64_t K, hipStream_t stream, int batch = 1,
                int64_t step_a = 0, int64_t step_b = 0, int64_t step_c = 0)
{
    GemmArgs g{};
    g.A = A;
    g.B = B;
    g.C = C;
    g.M = (int)M;
    g.N = (int)N;
    g.K = (int)K;
    g.lda = lda;
    g.ldb = ldb;
    g.ldc = ldc;
    g.batch = batch;
    g.batch_inner = 1;
    g.sAo = step_a;
    g.sBo = step_b;
    g.sCo = step_c;
    g.b_is_nk = nk;
    return launch_gemm(g, stream);
}

// Parts of equal length that k is cut into, each a product of a batch, for products with few tiles: where the split GEMM's estimate for the batch
// and the launch that joins its results (3 us and 5 TB/s) is 0.97 of that for the whole or less. (Blocks whose down product or dx lies between 0.9 and
// 0.97, whole / in parts, us: backward 777 and 1024 tokens of 1024 -> 2816 297 / 278, 344 / 325, 2048 640 / 606, its forward pass 283 / 267, backward 4096
// of 512 -> 1536 397 / 377; forward 4096 of 640 -> 2560 318 / 324.) A function of the extents alone.
int parts_of_k(int64_t M, int64_t N, int64_t K)
{
    auto estimate = [&](int64_t parts) {
        return gsplit::estimate_us(gsplit::kVariants[gsplit::choose_variant(M, N, K / parts, parts)], M, N, K / parts, parts) +
               (parts > 1 ? 3.0 + (double)(parts + 1) * (double)M * (double)N * 4.0 / 5e6 : 0.0);
    };
    int best = 1;
    double least = 0.97 * estimate(1);
    for (const int parts : {2, 3, 4, 6, 8})
        if (K % parts == 0 && K / parts >= 256 && estimate(parts) < least) {
            best = parts;
            least = estimate(parts);
        }
    return best;
}
size_t parts_bytes(int64_t M, int64_t N, int64_t K)
{
    const int n = parts_of_k(M, N, K);
    return n > 1 ? (size_t)n * M * N * 4 : 0;
}

// gemm() of which k may be cut, through `parts` (parts_bytes()).
hipError_t gemm_in_parts(const float* A, int64_t lda, const float* B, int64_t ldb, bool nk, float* C, int64_t ldc, int64_t M, int64_t N, int64_t K, float* parts, hipStream_t stream)
{
    const int n = parts_of_k(M, N, K);
    if (n == 1) return gemm(A, lda, B, ldb, nk, C, ldc, M, N, K, stream);
    const int64_t k = K / n;
    const hipError_t e = gemm(A, lda, B, ldb, nk, parts, N, M, N, k, stream, n, k, nk ? k : k * ldb, M * N);
    if (e != hipSuccess) return e;
    return launch_join(parts, n, C, ldc, M, N, stream);
}

// ---- few tokens

template <typename T, int TB, bool GATED, bool ALIGNED>
hipError_t launch_rows_as(const ffrows::Args& a, hipStream_t stream)
{
    static LdsLimit limit;
    // waves of a work-group: eight for each CU over all work-groups, as far as there are chunks for them
    const int groups = (a.N + 15) / 16, chunks = (int)(((int64_t)a.K * sizeof(T) + 127) / 128);
    int waves = 2;
    while (waves < (TB == 4 ? 8 : 16) && groups * waves < 2048 && 2 * waves <= chunks) waves *= 2;
    const size_t lds = (size_t)waves * TB * (GATED ? 2 : 1) * 256 * sizeof(float);
    auto* const kernel = ffrows::rows_kernel<T, TB, GATED, ALIGNED>;
    const hipError_t e = lds > 65536 ? raise_lds_limit(reinterpret_cast<const void*>(kernel), lds, limit) : hipSuccess;
    return e != hipSuccess ? e : launch_kernel(kernel, dim3(groups), dim3(64 * waves), lds, stream, a);
}

template <typename T, bool GATED>
hipError_t launch_rows(const ffrows::Args& a, bool aligned, hipStream_t stream)
{
    auto with = [&](auto tb) {
        constexpr int TB = decltype(tb)::value;
        return aligned ? launch_rows_as<T, TB, GATED, true>(a, stream) : launch_rows_as<T, TB, GATED, false>(a, stream);
    };
    if (a.T <= 16) return with(std::integral_constant<int, 1>{});
    if (a.T <= 32) return with(std::integral_constant<int, 2>{});
    return with(std::integral_constant<int, 4>{});
}

// 16-bit operands whose rows are no whole 16-byte units are copied first, to rows that are, with zeros behind their ends: 1024 tokens 1001 -> 2777
// took 175 us with loads of single elements where they are used, 76 so.
struct Copy {
    const void* in;
    int64_t ld, R, C;
    void* out;
    int64_t ld_out;
};
struct Copies {
    Copy c[5];
};
template <typename T>
__global__ __launch_bounds__(kThreads) void copy_rows_kernel(const Copies all)
{
    constexpr int E = 16 / (int)sizeof(T);
    const Copy& c = all.c[blockIdx.z];
    const T* const in = static_cast<const T*>(c.in);
    T* const out = static_cast<T*>(c.out);
    const int64_t units = c.ld_out / E;
    for (int64_t r = blockIdx.y; r < c.R; r += gridDim.y)
        for (int64_t u = (int64_t)blockIdx.x * kThreads + threadIdx.x; u < units; u += (int64_t)gridDim.x * kThreads) {
            struct __attribute__((packed, aligned(2))) Loose { Pack<T, E> v; };
            Pack<T, E> v;
            if (u * E + E <= c.C) {
                v = reinterpret_cast<const Loose*>(in + r * c.ld + u * E)->v;
            } else {
#pragma unroll
                for (int i = 0; i < E; ++i) v.v[i] = u * E + i < c.C ? in[r * c.ld + u * E + i] : from_float<T>(0.f);
            }
            *reinterpret_cast<Pack<T, E>*>(out + r * c.ld_out + u * E) = v;
        }
}

int64_t whole(int64_t n, int es) { return (n * es + 15) / 16 * 16 / es; }
// Whether a call copies its operands: by the descriptor alone (pointers that are not aligned take the kernels of single elements).
bool copies(const anr_gated_ff_desc& d, bool backward)
{
    const int es = element_bytes(d.dtype);
    for (const int64_t n : {d.C, d.F, d.ldx, d.ldw, d.ld_down, backward ? d.ldy : 0})
        if (n * es % 16 != 0) return true;
    return false;
}
// A call's arguments with the copies in place of the operands; `at`: where they go, at the end the first byte behind them.
struct Operands {
    const void *x, *dy, *w_gate, *w_up, *w_down;
    int64_t ldx, ldy, ldw, ld_down;
};
size_t copied_bytes(const anr_gated_ff_desc& d, bool backward)
{
    const size_t es = element_bytes(d.dtype), c = whole(d.C, (int)es), f = whole(d.F, (int)es);
    return whole_lines(d.T * c * es) * (backward ? 2 : 1) + 2 * whole_lines(d.F * c * es) + whole_lines(d.C * f * es);
}
hipError_t operands_of(const GatedFfArgs& g, bool backward, char* at, Operands* o, hipStream_t stream)
{
    const anr_gated_ff_desc& d = g.d;
    *o = {g.x, g.dy, g.w_gate, g.w_up, g.w_down, d.ldx, d.ldy, d.ldw, d.ld_down};
    if (!copies(d, backward)) return hipSuccess;
    const int es = element_bytes(d.dtype);
    Copies all{};
    unsigned n = 0;
    auto copy = [&](const void*& p, int64_t ld, int64_t R, int64_t C) {
        all.c[n++] = {p, ld, R, C, at, whole(C, es)};
        p = at;
        at += whole_lines((size_t)R * whole(C, es) * es);
    };
    copy(o->x, d.ldx, d.T, d.C);
    if (backward) copy(o->dy, d.ldy, d.T, d.C);
    copy(o->w_gate, d.ldw, d.F, d.C);
    copy(o->w_up, d.ldw, d.F, d.C);
    copy(o->w_down, d.ld_down, d.C, d.F);
    o->ldx = o->ldw = whole(d.C, es);
    if (backward) o->ldy = o->ldx;
    o->ld_down = whole(d.F, es);
    dim3 grid = grid_of(std::max(o->ldx, o->ld_down) * es / 16, kThreads, std::max({d.T, d.F, d.C}), 1);
    grid.z = n;
    return with_type(d.dtype, [&](auto t) { return launch_kernel(copy_rows_kernel<decltype(t)>, grid, dim3(kThreads), 0, stream, all); });
}
bool whole_rows(const void* p, int64_t ld, int es) { return is_aligned16(p) && ld * es % 16 == 0; }

hipError_t forward_few(const GatedFfArgs& g, hipStream_t stream)
{
    const anr_gated_ff_desc& d = g.d;
    const int es = element_bytes(d.dtype);
    const int64_t F8 = whole(d.F, es);
    auto units = [&](const void* p, int64_t ld, int64_t K) { return whole_rows(p, ld, es) && K * es % 16 == 0; };
    return with_type(d.dtype, [&](auto t) {
        using T = decltype(t);
        ffrows::Args a{};
        a.x = g.x;
        a.w[0] = g.w_gate;
        a.w[1] = g.w_up;
        a.d = g.ws;
        a.gate = g.gate;
        a.up = g.up;
        a.ldx = d.ldx;
        a.ldw[0] = a.ldw[1] = d.ldw;
        a.ldd = F8;
        a.whole_rows = true;
        a.ld_pre = d.ldpre;
        a.T = (int)d.T;
        a.N = (int)d.F;
        a.K = (int)d.C;
        a.act = d.act;
        const hipError_t e = launch_rows<T, true>(a, units(g.x, d.ldx, d.C) && units(g.w_gate, d.ldw, d.C) && units(g.w_up, d.ldw, d.C), stream);
        if (e != hipSuccess) return e;
        ffrows::Args b{};
        b.x = g.ws;
        b.w[0] = g.w_down;
        b.d = g.y;
        b.ldx = F8;
        b.ldw[0] = d.ld_down;
        b.ldd = d.ldy;
        b.T = (int)d.T;
        b.N = (int)d.C;
        b.K = (int)d.F;
        return launch_rows<T, false>(b, units(g.w_down, d.ld_down, d.F), stream);
    });
}

// ---- 16-bit products

mm16::Problem problem(const void* x, int64_t ldx, const void* w, int64_t ldw, void* d, int64_t ldd, int64_t M, int64_t N, int64_t K)
{
    mm16::Problem p{};
    p.x[0] = p.x[1] = x;
    p.w[0] = p.w[1] = w;
    p.d = d;
    p.ldx = ldx;
    p.ldw = ldw;
    p.ldd = ldd;
    p.M = (int)M;
    p.N = (int)N;
    p.K = (int)K;
    p.segments = 1;
    return p;
}

int64_t tiles_of(int64_t M, int64_t N, int tile_m, int tile_n) { return ((M + tile_m - 1) / tile_m) * ((N + tile_n - 1) / tile_n); }

int64_t chunks_of(int64_t K) { return (K + mm16::BK - 1) / mm16::BK; }

// The tile with the shortest estimated time: rounds of work-groups over the CUs, each with its chunks and ends (us). A tile of 256 takes a CU
// for itself, of those of 128 it takes two; one alone is split over two groups of waves. Measured (256 / 128 / 128 twice, 4096 tokens, 1024 -> 2816):
// gate and up, both stored, 72 / 72 / 88 us, down 61 / 32 / 30, hidden gradients 54 / 53 / 70, dx 111 / 62 / 54, weights 93 / 103 / 110; 8192 tokens, 4096 -> 11264:
// 1226 / 1568 / 1792, 564 / 745 / 835, 848 / 925 / 1175, 1142 / 1580 / 1682, 1851 / 2328 / 2492.
struct Choice {
    mm16::Shape shape;
    double us;
};
Choice choose_shape(int64_t tiles256, int64_t tiles128, int64_t chunks)
{
    const double large = (double)((tiles256 + 255) / 256) * (1.7 * (double)chunks + 4.0);
    const int64_t full = tiles128 / 512, rest = tiles128 % 512;
    const double pair = 1.14 * (double)chunks + 4.0, alone = 0.60 * (double)chunks + 4.0;
    const bool twice = tiles128 <= 256;
    const double small = twice ? alone : (double)full * pair + (rest > 256 ? pair : rest > 0 ? 0.75 * (double)chunks + 4.0 : 0.0);
    if (large < small) return {mm16::SHAPE_256, large};
    return {twice ? mm16::SHAPE_128_TWICE : mm16::SHAPE_128, small};
}

// Work-groups that share a tile's k, for products with few tiles: the number with the shortest estimated time, that of the launch that joins their
// sums among it. A function of the extents alone.
int splits_of(int64_t M, int64_t N, int64_t chunks)
{
    int best = 1;
    double least = choose_shape(tiles_of(M, N, 256, 256), tiles_of(M, N, 128, 128), chunks).us;
    for (int s = 2; s <= 16 && chunks / s >= 4; ++s) {
        const double us = choose_shape(s * tiles_of(M, N, 256, 256), s * tiles_of(M, N, 128, 128), (chunks + s - 1) / s).us + 4.0 + 2.0 * s * (double)M * (double)N * 4.0 / 8e6;
        if (us < least) {
            least = us;
            best = s;
        }
    }
    return best;
}

hipError_t launch(mm16::Form form, int dtype, bool aligned, mm16::Args& a, hipStream_t stream)
{
    const int n_share = form == mm16::FORM_GATED ? 2 : 1;
    auto tiles = [&](int edge) {
        int64_t n = 0;
        for (int i = 0; i < a.problems; ++i) n += tiles_of(a.p[i].M, a.p[i].N, edge, edge / n_share);
        return n * a.splits;
    };
    const mm16::Shape shape = choose_shape(tiles(256), tiles(128), chunks_of(a.p[0].K) * a.p[0].segments / a.splits).shape;
    const int tile = mm16::edge_of(shape);
    a.first_tile[0] = 0;
    for (int i = 0; i < a.problems; ++i) {
        a.p[i].tiles_m = (a.p[i].M + tile - 1) / tile;
        a.p[i].tiles_n = (a.p[i].N + tile / n_share - 1) / (tile / n_share);
        a.first_tile[i + 1] = a.first_tile[i] + a.p[i].tiles_m * a.p[i].tiles_n;
    }
    a.band = 8;
    return dtype == ANR_F16 ? mm16::launch_products_f16(form, shape, aligned, a, stream) : mm16::launch_products_bf16(form, shape, aligned, a, stream);
}

// A product whose k may be shared: through `parts` where it is.
hipError_t launch_shared(mm16::Form form, int dtype, bool aligned, const mm16::Problem& p, int splits, float* parts, hipStream_t stream)
{
    mm16::Args a{};
    a.p[0] = p;
    a.problems = 1;
    a.splits = splits;
    if (splits > 1) a.p[0].d = parts;
    hipError_t e = launch(form, dtype, aligned, a, stream);
    if (e != hipSuccess || splits == 1) return e;
    return with_type(dtype, [&](auto t) {
        using T = decltype(t);
        return launch_join(parts, splits, static_cast<T*>(p.d), p.ldd, p.M, p.N, stream);
    });
}

hipError_t forward_16(const GatedFfArgs& g, hipStream_t stream)
{
    const anr_gated_ff_desc& d = g.d;
    const int64_t F8 = whole(d.F, 2);
    char* const ws = static_cast<char*>(g.ws);
    const int splits = splits_of(d.T, d.C, chunks_of(d.F));
    char* const parts = ws + whole_lines((size_t)d.T * F8 * 2);
    Operands o;
    hipError_t e = operands_of(g, false, parts + whole_lines(splits > 1 ? (size_t)splits * d.T * d.C * 4 : 0), &o, stream);
    if (e != hipSuccess) return e;
    mm16::Args a{};
    a.p[0] = problem(o.x, o.ldx, o.w_gate, o.ldw, ws, F8, d.T, d.F, d.C);
    a.p[0].w[1] = o.w_up;
    a.problems = a.splits = 1;
    a.act = d.act;
    a.gate = g.gate;
    a.up = g.up;
    a.ld_pre = d.ldpre;
    a.whole_rows = true;
    e = launch(mm16::FORM_GATED, d.dtype, whole_rows(o.x, o.ldx, 2) && whole_rows(o.w_gate, o.ldw, 2) && whole_rows(o.w_up, o.ldw, 2), a, stream);
    if (e != hipSuccess) return e;
    const mm16::Problem down = problem(ws, F8, o.w_down, o.ld_down, g.y, d.ldy, d.T, d.C, d.F);
    return launch_shared(mm16::FORM_ROWS, d.dtype, whole_rows(o.w_down, o.ld_down, 2), down, splits, reinterpret_cast<float*>(parts), stream);
}

hipError_t backward_16(const GatedFfArgs& g, hipStream_t stream)
{
    const anr_gated_ff_desc& d = g.d;
    const int64_t T = d.T, C = d.C, F = d.F, F8 = whole(F, 2);
    char* const dg = static_cast<char*>(g.ws);
    char* const du = dg + 2 * F8;                       // side by side: rows of 2 F8
    char* const h = dg + whole_lines((size_t)T * F8 * 4);
    char* const parts = h + whole_lines((size_t)T * F8 * 2);
    const int splits = splits_of(T, C, 2 * chunks_of(F));
    Operands o;
    hipError_t e = operands_of(g, true, parts + whole_lines(splits > 1 ? (size_t)splits * T * C * 4 : 0), &o, stream);
    if (e != hipSuccess) return e;
    const bool aligned_w = whole_rows(o.w_gate, o.ldw, 2) && whole_rows(o.w_up, o.ldw, 2), aligned_dy = whole_rows(o.dy, o.ldy, 2), aligned_x = whole_rows(o.x, o.ldx, 2);
    mm16::Args a{};
    a.p[0] = problem(o.dy, o.ldy, o.w_down, o.ld_down, dg, 2 * F8, T, F, C);
    a.problems = a.splits = 1;
    a.act = d.act;
    a.gate = g.gate;
    a.up = g.up;
    a.ld_pre = d.ldpre;
    a.du = du;
    a.h = h;
    a.ld_h = F8;
    a.whole_rows = true;
    e = launch(mm16::FORM_HIDDEN_GRADS, d.dtype, aligned_dy && whole_rows(o.w_down, o.ld_down, 2), a, stream);
    if (e == hipSuccess && g.dx) {
        mm16::Problem p = problem(dg, 2 * F8, o.w_gate, o.ldw, g.dx, d.lddx, T, C, F);
        p.x[1] = du;
        p.w[1] = o.w_up;
        p.segments = 2;
        e = launch_shared(mm16::FORM_INPUT_GRAD, d.dtype, aligned_w, p, splits, reinterpret_cast<float*>(parts), stream);
    }
    if (e != hipSuccess || !(g.dw_gate || g.dw_up || g.dw_down)) return e;
    mm16::Args b{};
    b.splits = 1;
    if (g.dw_gate) b.p[b.problems++] = problem(dg, 2 * F8, o.x, o.ldx, g.dw_gate, d.lddw, F, C, T);
    if (g.dw_up) b.p[b.problems++] = problem(du, 2 * F8, o.x, o.ldx, g.dw_up, d.lddw, F, C, T);
    if (g.dw_down) b.p[b.problems++] = problem(o.dy, o.ldy, h, F8, g.dw_down, d.ld_ddown, C, F, T);
    return launch(mm16::FORM_WEIGHT_GRADS, d.dtype, (aligned_x || !(g.dw_gate || g.dw_up)) && (aligned_dy || !g.dw_down), b, stream);
}

// ---- float32 products

// Gate, up, activation and product in one launch: what it multiplies, and whether it runs, by the descriptor alone.
GatedGemmArgs gated_product(const anr_gated_ff_desc& d)
{
    GatedGemmArgs a{};
    a.M = (int)d.T;
    a.N = (int)d.F;
    a.K = (int)d.C;
    a.lda = d.ldx;
    a.ldb = d.ldw;
    a.ldc = d.F;
    a.batch = a.batch_inner = 1;
    a.b_is_nk = true;
    a.ld_pre = d.ldpre;
    a.act = d.act;
    return a;
}
// Of the workspace: h, and gate and up where they are products of their own.
int hidden_matrices(const anr_gated_ff_desc& d) { return gemm_split_gated_takes(gated_product(d)) ? 1 : 3; }

hipError_t forward_32(const GatedFfArgs& g, hipStream_t stream)
{
    const anr_gated_ff_desc& d = g.d;
    const size_t tf = whole_lines((size_t)d.T * d.F * 4) / 4;
    float* const h = static_cast<float*>(g.ws);
    GatedGemmArgs a = gated_product(d);
    a.A = static_cast<const float*>(g.x);
    a.B = static_cast<const float*>(g.w_gate);
    a.B2 = static_cast<const float*>(g.w_up);
    a.C = h;
    a.gate = static_cast<float*>(g.gate);
    a.up = static_cast<float*>(g.up);
    hipError_t e = hipSuccess;
    if (hidden_matrices(d) == 1) {
        e = launch_gemm_split_gated(a, stream);
    } else {
        float* const gate = g.gate ? a.gate : h + tf;
        float* const up = g.gate ? a.up : h + 2 * tf;
        const int64_t ld = g.gate ? d.ldpre : d.F;
        e = gemm(a.A, d.ldx, a.B, d.ldw, true, gate, ld, d.T, d.F, d.C, stream);
        if (e == hipSuccess) e = gemm(a.A, d.ldx, a.B2, d.ldw, true, up, ld, d.T, d.F, d.C, stream);
        if (e == hipSuccess)
            e = with_activation(d.act, [&](auto act) {
                return launch_kernel(product_of_gate_kernel<decltype(act)::value>, grid_of(d.F, kThreads, d.T, 1), dim3(kThreads), 0, stream, static_cast<const float*>(gate),
                                     static_cast<const float*>(up), ld, h, d.T, d.F);
            });
    }
    if (e != hipSuccess) return e;
    return gemm_in_parts(h, d.F, static_cast<const float*>(g.w_down), d.ld_down, true, static_cast<float*>(g.y), d.ldy, d.T, d.C, d.F, h + hidden_matrices(d) * tf, stream);
}

hipError_t backward_32(const GatedFfArgs& g, hipStream_t stream)
{
    const anr_gated_ff_desc& d = g.d;
    const int64_t T = d.T, C = d.C, F = d.F;
    const size_t tf = whole_lines((size_t)T * F * 4) / 4;
    float* const dh = static_cast<float*>(g.ws);
    float* const h = dh + tf;
    float* const dgu = h + tf;                          // [T, 2F]
    float* const turned = dgu + 2 * tf;                 // [2F, T]
    float* const weights = turned + 2 * tf;             // [2F, C], gate's and up's
    float* const dy_turned = weights + whole_lines((size_t)F * C * 8) / 4;
    float* const parts = dy_turned + whole_lines((size_t)T * C * 4) / 4;
    const float *const dy = static_cast<const float*>(g.dy), *const x = static_cast<const float*>(g.x);
    const float *const wg = static_cast<const float*>(g.w_gate), *const wu = static_cast<const float*>(g.w_up);
    const bool one_tensor = wu == wg + F * d.ldw;       // (gate's and up's weights are rows of one matrix)
    hipError_t e = gemm(dy, d.ldy, static_cast<const float*>(g.w_down), d.ld_down, false, dh, F, T, F, C, stream);
    if (e == hipSuccess)
        e = with_activation(d.act, [&](auto act) {
            return launch_kernel(hidden_gradients_kernel<decltype(act)::value>, grid_of(F, 32, T, 32), dim3(kThreads), 0, stream, static_cast<const float*>(dh),
                                 static_cast<const float*>(g.gate), static_cast<const float*>(g.up), d.ldpre, dgu, turned, h, T, F);
        });
    Layouts l{};
    unsigned n = 0;
    if (g.dx && !one_tensor) {
        l.l[n++] = {wg, d.ldw, F, C, weights, false};
        l.l[n++] = {wu, d.ldw, F, C, weights + F * C, false};
    }
    if (g.dw_down) l.l[n++] = {dy, d.ldy, T, C, dy_turned, true};
    if (e == hipSuccess && n > 0) {
        dim3 grid = grid_of(C, 32, std::max(T, F), 32);
        grid.z = n;
        e = launch_kernel(lay_out_kernel, grid, dim3(kThreads), 0, stream, l);
    }
    if (e == hipSuccess && g.dx)
        e = gemm_in_parts(dgu, 2 * F, one_tensor ? wg : weights, one_tensor ? d.ldw : C, false, static_cast<float*>(g.dx), d.lddx, T, C, 2 * F, parts, stream);
    float *const dwg = static_cast<float*>(g.dw_gate), *const dwu = static_cast<float*>(g.dw_up);
    if (e == hipSuccess && dwg && dwu) {                // two products of one launch
        e = gemm(turned, T, x, d.ldx, false, dwg, d.lddw, F, C, T, stream, 2, F * T, 0, dwu - dwg);
    } else if (e == hipSuccess && (dwg || dwu)) {
        e = gemm(dwg ? turned : turned + F * T, T, x, d.ldx, false, dwg ? dwg : dwu, d.lddw, F, C, T, stream);
    }
    if (e == hipSuccess && g.dw_down) e = gemm(dy_turned, T, h, F, false, static_cast<float*>(g.dw_down), d.ld_ddown, C, F, T, stream);
    return e;
}

}  // namespace

size_t gated_ff_workspace_bytes(const GatedFfArgs& g, bool backward)
{
    const anr_gated_ff_desc& d = g.d;
    const size_t T = (size_t)d.T, C = (size_t)d.C, F = (size_t)d.F;
    if (T == 0) return 0;
    const size_t es = element_bytes(d.dtype), tf = whole_lines(T * whole(d.F, (int)es) * es);
    if (!backward && few_tokens(d)) return tf;
    if (d.dtype == ANR_F32) {
        if (backward) return 6 * tf + whole_lines(F * C * 8) + whole_lines(T * C * 4) + parts_bytes(d.T, d.C, 2 * d.F);
        return hidden_matrices(d) * tf + parts_bytes(d.T, d.C, d.F);
    }
    const int splits = splits_of(d.T, d.C, (backward ? 2 : 1) * chunks_of(d.F));
    const size_t parts = whole_lines(splits > 1 ? (size_t)splits * T * C * 4 : 0), copied = copies(d, backward) ? copied_bytes(d, backward) : 0;
    return (backward ? whole_lines(T * whole(d.F, 2) * 4) : 0) + tf + parts + copied;
}

hipError_t launch_gated_ff(const GatedFfArgs& g, hipStream_t stream)
{
    if (g.d.T == 0) return hipSuccess;
    if (few_tokens(g.d)) return forward_few(g, stream);
    return g.d.dtype == ANR_F32 ? forward_32(g, stream) : forward_16(g, stream);
}

hipError_t launch_gated_ff_backward(const GatedFfArgs& g, hipStream_t stream)
{
    const anr_gated_ff_desc& d = g.d;
    if (d.T > 0) return d.dtype == ANR_F32 ? backward_32(g, stream) : backward_16(g, stream);
    hipError_t e = hipSuccess;
    auto zero = [&](void* p, int64_t ld, int64_t M, int64_t N) {
        if (e == hipSuccess && p)
            e = with_type(d.dtype, [&](auto t) {
                using T = decltype(t);
                return launch_kernel(zero_kernel<T>, grid_of(N, kThreads, M, 1), dim3(kThreads), 0, stream, static_cast<T*>(p), ld, M, N);
            });
    };
    zero(g.dw_gate, d.lddw, d.F, d.C);
    zero(g.dw_up, d.lddw, d.F, d.C);
    zero(g.dw_down, d.ld_ddown, d.C, d.F);
    return e;
}

}  // namespace anr
