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
constexpr int kFewTokens = 64;                  // at most four blocks of sixteen (ff_rows_kernel.h)

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

// D [M,N] in T = the sum of the `splits` packed matrices at `parts`.
template <typename T>
__global__ __launch_bounds__(kThreads) void join_kernel(const float* parts, int splits, T* d, int64_t ldd, int64_t M, int64_t N)
{
    for (int64_t m = blockIdx.y; m < M; m += gridDim.y)
        for (int64_t n = (int64_t)blockIdx.x * kThreads + threadIdx.x; n < N; n += (int64_t)gridDim.x * kThreads) {
            float sum = 0.f;
            for (int s = 0; s < splits; ++s) sum += parts[((int64_t)s * M + m) * N + n];
            d[m * ldd + n] = from_float<T>(sum);
        }
}

template <typename T>
__global__ __launch_bounds__(kThreads) void zero_kernel(T* d, int64_t ldd, int64_t M, int64_t N)
{
    for (int64_t m = blockIdx.y; m < M; m += gridDim.y)
        for (int64_t n = (int64_t)blockIdx.x * kThreads + threadIdx.x; n < N; n += (int64_t)gridDim.x * kThreads) d[m * ldd + n] = T(0.f);
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
// and the launch that joins its results (3 us and 5 TB/s) is 0.9 of that for the whole or less. A function of the extents alone.
int parts_of_k(int64_t M, int64_t N, int64_t K)
{
    auto estimate = [&](int64_t parts) {
        return gsplit::estimate_us(gsplit::kVariants[gsplit::choose_variant(M, N, K / parts, parts)], M, N, K / parts, parts) +
               (parts > 1 ? 3.0 + (double)(parts + 1) * (double)M * (double)N * 4.0 / 5e6 : 0.0);
    };
    int best = 1;
    double least = 0.9 * estimate(1);
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
    return launch_kernel(join_kernel<float>, grid_of(N, kThreads, M, 1), dim3(kThreads), 0, stream, static_cast<const float*>(parts), n, C, ldc, M, N);
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

// 16-byte units: pointer, leading dimension and extent.
bool whole_units(const void* p, int64_t ld, int64_t extent, int es) { return is_aligned16(p) && ld * es % 16 == 0 && extent * es % 16 == 0; }

hipError_t forward_few(const GatedFfArgs& g, hipStream_t stream)
{
    const anr_gated_ff_desc& d = g.d;
    const int es = element_bytes(d.dtype);
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
        a.ldd = d.F;
        a.ld_pre = d.ldpre;
        a.T = (int)d.T;
        a.N = (int)d.F;
        a.K = (int)d.C;
        a.act = d.act;
        hipError_t e = launch_rows<T, true>(a, whole_units(g.x, d.ldx, d.C, es) && whole_units(g.w_gate, d.ldw, d.C, es) && whole_units(g.w_up, d.ldw, d.C, es), stream);
        if (e != hipSuccess) return e;
        ffrows::Args b{};
        b.x = g.ws;
        b.w[0] = g.w_down;
        b.d = g.y;
        b.ldx = d.F;
        b.ldw[0] = d.ld_down;
        b.ldd = d.ldy;
        b.T = (int)d.T;
        b.N = (int)d.C;
        b.K = (int)d.F;
        return launch_rows<T, false>(b, whole_units(g.ws, d.F, d.F, es) && whole_units(g.w_down, d.ld_down, d.F, es), stream);
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

// Work-groups that share a tile's k, for products with fewer tiles than CUs: as many as fill them, with four chunks each or more.
int splits_of(int64_t M, int64_t N, int64_t chunks)
{
    const int64_t tiles = tiles_of(M, N, 128, 128);
    if (tiles >= 256) return 1;
    return (int)std::max<int64_t>(1, std::min<int64_t>({(512 + tiles - 1) / tiles, chunks / 4, 16}));
}

int64_t chunks_of(int64_t K) { return (K + mm16::BK - 1) / mm16::BK; }

// The tile with the shortest estimated time: rounds of work-groups over the CUs, each with its chunks and ends (us). A tile of 256 takes a CU
// for itself, of those of 128 it takes two; one alone is split over two groups of waves.
mm16::Shape choose_shape(int64_t tiles256, int64_t tiles128, int64_t chunks)
{
    const double large = (double)((tiles256 + 255) / 256) * (1.7 * (double)chunks + 4.0);
    const int64_t full = tiles128 / 512, rest = tiles128 % 512;
    const double pair = 1.14 * (double)chunks + 4.0, alone = 0.60 * (double)chunks + 4.0;
    if (tiles128 <= 256) return large < alone ? mm16::SHAPE_256 : mm16::SHAPE_128_TWICE;
    const double small = (double)full * pair + (rest > 256 ? pair : rest > 0 ? 0.75 * (double)chunks + 4.0 : 0.0);
    return large < small ? mm16::SHAPE_256 : mm16::SHAPE_128;
}

hipError_t launch(mm16::Form form, int dtype, bool aligned, mm16::Args& a, hipStream_t stream)
{
    const int n_share = form == mm16::FORM_GATED ? 2 : 1;
    auto tiles = [&](int edge) {
        int64_t n = 0;
        for (int i = 0; i < a.problems; ++i) n += tiles_of(a.p[i].M, a.p[i].N, edge, edge / n_share);
        return n * a.splits;
    };
    const mm16::Shape shape = choose_shape(tiles(256), tiles(128), chunks_of(a.p[0].K) * a.p[0].segments / a.splits);
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
        return launch_kernel(join_kernel<T>, grid_of(p.N, kThreads, p.M, 1), dim3(kThreads), 0, stream, parts, splits, static_cast<T*>(p.d), p.ldd, (int64_t)p.M, (int64_t)p.N);
    });
}

hipError_t forward_16(const GatedFfArgs& g, hipStream_t stream)
{
    const anr_gated_ff_desc& d = g.d;
    char* const ws = static_cast<char*>(g.ws);
    mm16::Args a{};
    a.p[0] = problem(g.x, d.ldx, g.w_gate, d.ldw, ws, d.F, d.T, d.F, d.C);
    a.p[0].w[1] = g.w_up;
    a.problems = a.splits = 1;
    a.act = d.act;
    a.gate = g.gate;
    a.up = g.up;
    a.ld_pre = d.ldpre;
    const bool aligned = whole_units(g.x, d.ldx, d.C, 2) && whole_units(g.w_gate, d.ldw, d.C, 2) && whole_units(g.w_up, d.ldw, d.C, 2);
    hipError_t e = launch(mm16::FORM_GATED, d.dtype, aligned, a, stream);
    if (e != hipSuccess) return e;
    const mm16::Problem down = problem(ws, d.F, g.w_down, d.ld_down, g.y, d.ldy, d.T, d.C, d.F);
    return launch_shared(mm16::FORM_ROWS, d.dtype, whole_units(ws, d.F, d.F, 2) && whole_units(g.w_down, d.ld_down, d.F, 2), down, splits_of(d.T, d.C, chunks_of(d.F)),
                         reinterpret_cast<float*>(ws + whole_lines((size_t)d.T * d.F * 2)), stream);
}

hipError_t backward_16(const GatedFfArgs& g, hipStream_t stream)
{
    const anr_gated_ff_desc& d = g.d;
    const int64_t T = d.T, C = d.C, F = d.F;
    char* const dg = static_cast<char*>(g.ws);
    char* const du = dg + 2 * F;                        // side by side: rows of 2 F
    char* const h = dg + whole_lines((size_t)T * F * 4);
    float* const parts = reinterpret_cast<float*>(h + whole_lines((size_t)T * F * 2));
    mm16::Args a{};
    a.p[0] = problem(g.dy, d.ldy, g.w_down, d.ld_down, dg, 2 * F, T, F, C);
    a.problems = a.splits = 1;
    a.act = d.act;
    a.gate = g.gate;
    a.up = g.up;
    a.ld_pre = d.ldpre;
    a.du = du;
    a.h = h;
    a.ld_h = F;
    hipError_t e = launch(mm16::FORM_HIDDEN_GRADS, d.dtype, whole_units(g.dy, d.ldy, C, 2) && whole_units(g.w_down, d.ld_down, F, 2), a, stream);
    if (e == hipSuccess && g.dx) {
        mm16::Problem p = problem(dg, 2 * F, g.w_gate, d.ldw, g.dx, d.lddx, T, C, F);
        p.x[1] = du;
        p.w[1] = g.w_up;
        p.segments = 2;
        const bool aligned = F % 8 == 0 && whole_units(g.w_gate, d.ldw, C, 2) && whole_units(g.w_up, d.ldw, C, 2);
        e = launch_shared(mm16::FORM_INPUT_GRAD, d.dtype, aligned, p, splits_of(T, C, 2 * chunks_of(F)), parts, stream);
    }
    if (e != hipSuccess || !(g.dw_gate || g.dw_up || g.dw_down)) return e;
    mm16::Args b{};
    b.splits = 1;
    bool aligned = F % 8 == 0 && C % 8 == 0;
    if (g.dw_gate) b.p[b.problems++] = problem(dg, 2 * F, g.x, d.ldx, g.dw_gate, d.lddw, F, C, T);
    if (g.dw_up) b.p[b.problems++] = problem(du, 2 * F, g.x, d.ldx, g.dw_up, d.lddw, F, C, T);
    if (g.dw_gate || g.dw_up) aligned = aligned && whole_units(g.x, d.ldx, C, 2);
    if (g.dw_down) {
        b.p[b.problems++] = problem(g.dy, d.ldy, h, F, g.dw_down, d.ld_ddown, C, F, T);
        aligned = aligned && whole_units(g.dy, d.ldy, C, 2);
    }
    return launch(mm16::FORM_WEIGHT_GRADS, d.dtype, aligned, b, stream);
}

// ---- float32 products

hipError_t forward_32(const GatedFfArgs& g, hipStream_t stream)
{
    const anr_gated_ff_desc& d = g.d;
    const size_t tf = whole_lines((size_t)d.T * d.F * 4) / 4;
    float* const h = static_cast<float*>(g.ws);
    GatedGemmArgs a{};
    a.A = static_cast<const float*>(g.x);
    a.B = static_cast<const float*>(g.w_gate);
    a.B2 = static_cast<const float*>(g.w_up);
    a.C = h;
    a.M = (int)d.T;
    a.N = (int)d.F;
    a.K = (int)d.C;
    a.lda = d.ldx;
    a.ldb = d.ldw;
    a.ldc = d.F;
    a.batch = a.batch_inner = 1;
    a.b_is_nk = true;
    a.gate = static_cast<float*>(g.gate);
    a.up = static_cast<float*>(g.up);
    a.ld_pre = d.ldpre;
    a.act = d.act;
    hipError_t e = hipSuccess;
    if (gemm_split_gated_takes(a)) {
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
    return gemm_in_parts(h, d.F, static_cast<const float*>(g.w_down), d.ld_down, true, static_cast<float*>(g.y), d.ldy, d.T, d.C, d.F, h + 3 * tf, stream);
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
    if (d.dtype == ANR_F32) {
        const size_t tf = whole_lines(T * F * 4);
        if (backward) return 6 * tf + whole_lines(F * C * 8) + whole_lines(T * C * 4) + parts_bytes(d.T, d.C, 2 * d.F);
        return T <= kFewTokens ? tf : 3 * tf + parts_bytes(d.T, d.C, d.F);
    }
    const size_t tf = whole_lines(T * F * 2);
    const int splits = splits_of(d.T, d.C, (backward ? 2 : 1) * chunks_of(d.F));
    const size_t parts = splits > 1 ? (size_t)splits * T * C * 4 : 0;
    if (backward) return whole_lines(T * F * 4) + tf + parts;
    return T <= kFewTokens ? tf : tf + parts;
}

hipError_t launch_gated_ff(const GatedFfArgs& g, hipStream_t stream)
{
    if (g.d.T == 0) return hipSuccess;
    if (g.d.T <= kFewTokens) return forward_few(g, stream);
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
