// Root-mean-square norm (rms_norm_kernel.h): which kernels a call runs.
#include <algorithm>

#include "blocks_internal.h"
#include "rms_norm_kernel.h"
#include "rows_launch.h"

namespace anr {
namespace {

using rmsnorm::Args;
using rows::Plan;

constexpr int kMostGroups = 1 << 20;             // of a launch: rows beyond them are taken in turn

template <typename F>
hipError_t with_types(const RmsNormArgs& a, F f)
{
    return with_type(a.d.dtype, [&](auto t) {
        using T = decltype(t);
        if (a.d.param_dtype == ANR_F32) return f(t, 0.f);
        return f(t, T{});
    });
}

template <typename T>
Plan plan(const anr_rms_norm_desc& d) { return rows::plan_for<T>(d.C, d.T); }

Args arguments(const RmsNormArgs& g)
{
    Args a{};
    a.x = g.x;
    a.gamma = g.gamma;
    a.T = g.d.T;
    a.C = (int)g.d.C;
    a.ldx = g.d.ldx;
    a.ld_residual = g.d.ld_residual;
    a.ldh = g.d.ldh;
    a.ldy = g.d.ldy;
    return a;
}

template <bool QUANTIZED>
hipError_t launch_forward(const RmsNormArgs& g, hipStream_t stream)
{
    if (g.d.T == 0) return hipSuccess;
    Args a = arguments(g);
    a.residual = g.residual;
    a.h = g.h;
    a.y = g.y;
    a.eps = g.eps;
    a.rstd = g.rstd;
    a.scale = g.scale;
    return with_types(g, [&](auto t, auto p) {
        using T = decltype(t);
        using P = decltype(p);
        const Plan of = plan<T>(g.d);
        return rows::with_rows<T>(g.d.C, of, [&](auto v, auto u, auto whole) {
            constexpr int V = decltype(v)::value, U = decltype(u)::value;
            constexpr bool WHOLE = decltype(whole)::value;
            a.streaming = V > 1;
            const int64_t groups = std::min<int64_t>((a.T + of.rows - 1) / of.rows, kMostGroups);
            return launch_kernel(rmsnorm::forward_kernel<T, P, V, U, WHOLE, QUANTIZED, 1024>, dim3((unsigned)groups), dim3(of.threads, of.rows), 0, stream, a);
        });
    });
}

int64_t lines(const anr_rms_norm_desc& d)
{
    return with_type(d.dtype, [&](auto t) { return rows::backward_plan_for<decltype(t)>(d.C, d.T).lines; });
}

}  // namespace

size_t rms_norm_backward_workspace_bytes(const RmsNormArgs& g) { return g.d.T == 0 ? 0 : (size_t)lines(g.d) * g.d.C * sizeof(float); }

hipError_t launch_rms_norm(const RmsNormArgs& g, hipStream_t stream) { return launch_forward<false>(g, stream); }
hipError_t launch_rms_norm_q8(const RmsNormArgs& g, hipStream_t stream) { return launch_forward<true>(g, stream); }

hipError_t launch_rms_norm_backward(const RmsNormArgs& g, hipStream_t stream)
{
    Args a = arguments(g);
    a.dy = g.dy;
    a.dh = g.residual;
    a.h = g.h;
    a.rstd_in = g.rstd;
    a.sums = g.dgamma ? static_cast<float*>(g.ws) : nullptr;
    const int es = element_bytes(g.d.dtype), n = g.d.T == 0 ? 0 : (int)lines(g.d);
    if (n > 0) {
        const hipError_t e = with_types(g, [&](auto t, auto p) {
            using T = decltype(t);
            using P = decltype(p);
            const Plan of = rows::backward_plan_for<T>(g.d.C, g.d.T).rows;
            return rows::with_rows<T>(g.d.C, of, [&](auto v, auto u, auto whole) {
                constexpr int V = decltype(v)::value, U = decltype(u)::value;
                constexpr bool WHOLE = decltype(whole)::value;
                // (4096 x 9001 bf16 with the residual's gradient 104 us by ordinary stores, 117 past L2; 4096 x 4003 42.4, 38.7)
                a.streaming = V > 1 && (U == 1 || (is_aligned16(a.h) && a.ldh * es % 16 == 0));
                static LdsLimit limit;
                void (*const kernel)(Args) = rmsnorm::backward_kernel<T, P, V, U, WHOLE, 1024>;
                size_t lds = of.rows > 1 ? (size_t)of.rows * g.d.C * sizeof(float) : 0;
                if (rmsnorm::sums_apart(U * V)) {
                    lds = (size_t)U * V * rows::kMostThreads * sizeof(float);
                    const hipError_t e = raise_lds_limit(reinterpret_cast<const void*>(kernel), lds, limit);
                    if (e != hipSuccess) return e;
                }
                return launch_kernel(kernel, dim3((unsigned)n), dim3(of.threads, of.rows), lds, stream, a);
            });
        });
        if (e != hipSuccess) return e;
    }
    if (!g.dgamma) return hipSuccess;
    const unsigned groups = (unsigned)((g.d.C + rmsnorm::kJoinColumns - 1) / rmsnorm::kJoinColumns);
    return with_type(g.d.param_dtype, [&](auto p) {
        using P = decltype(p);
        return launch_kernel(rmsnorm::join_kernel<P>, dim3(groups), dim3(rmsnorm::kJoinColumns * rmsnorm::kJoinRuns), 0, stream, static_cast<const float*>(g.ws), n, (int)g.d.C,
                             static_cast<P*>(g.dgamma));
    });
}

}  // namespace anr
