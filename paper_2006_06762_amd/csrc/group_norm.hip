// Plan and launches of the group norm (group_norm_kernel.h).
#include "group_norm_kernel.h"

#include <algorithm>

#include "blocks_internal.h"

namespace anr {
namespace {

using namespace gnorm;

// The plan: a function of the descriptor and the pointers' alignment; the workspace it needs is a function of the
// descriptor alone (the most that either alignment takes).
struct Plan {
    Args args;
    Division d;
    bool vector;                    // 16-byte loads
    size_t bytes;                   // of workspace
};

// Strides that keep 16-byte units whole.
bool whole_units(const void* p, const int64_t* s, int V) { return is_aligned16(p) && s[0] % V == 0 && s[1] % V == 0 && s[2] % V == 0; }

Plan make_plan_with(const GroupNormArgs& g, bool backward, bool vector)
{
    Plan p{};
    Args& a = p.args;
    a.x = g.x;
    a.dy = g.dy;
    a.y = g.y;
    a.gamma = g.gamma;
    a.beta = g.beta;
    a.dgamma = g.dgamma;
    a.dbeta = g.dbeta;
    a.mean = g.mean;
    a.rstd = g.rstd;
    a.eps = g.eps;
    a.N = g.N;
    a.C = g.C;
    a.groups = g.groups;
    a.cg = g.C / g.groups;
    a.param_dtype = g.param_dtype;
    a.HW = g.H * g.W;
    auto pixels = [](const int64_t* s) { return Pixels{s[0], s[1], s[2]}; };
    a.px = pixels(g.xs);
    a.pdy = pixels(g.dys);
    a.py = pixels(g.ys);
    auto flat = [&](const int64_t* s) { return g.H == 1 || s[1] == (int64_t)g.W * s[2]; };
    a.flat = flat(g.xs) && (!backward || flat(g.dys)) && flat(g.ys);
    a.W = g.W;
    a.by_w = make_fastdiv(g.W);
    a.by_cg = make_fastdiv(a.cg);
    a.by_each = make_fastdiv(a.cg % kHeldChannels == 0 ? a.cg / kHeldChannels : a.cg);

    const int es = element_bytes(g.dtype), line = 128 / es;
    p.vector = vector;
    p.d = divide({g.N, a.HW, g.C, g.groups, es, vector, backward});
    a.chunk = p.d.chunk;
    a.halves = p.d.halves;
    a.slabs = p.d.slabs;
    a.slab_pixels = p.d.slab_pixels;
    // Stores past L2 wherever they are whole lines, small outputs too. Forward, so / not, alone and with a product over 512 (float32 256) channels that reads the
    // result: bf16 4 x 64^2 x 512 15.0 / 16.0, 31.9 / 31.7, 16 x 64^2 40.1 / 47.7, 98.4 / 94.9, 8 x 128^2 77.5 / 89.5, 179 / 186; float32 4 x 128^2 x 256 38.9 / 47.6,
    // 113.4 / 112.8.
    a.streaming = a.chunk % line == 0 && (reinterpret_cast<uintptr_t>(g.y) & 127) == 0 && g.ys[0] % line == 0 && g.ys[1] % line == 0 && g.ys[2] % line == 0;
    a.values = (double)a.HW * (double)a.cg;
    if (backward) {
        const size_t of_groups = p.d.resident ? 0 : 2 * (size_t)g.N * a.slabs * g.groups;
        p.bytes = sizeof(float) * (of_groups + 2 * (size_t)g.N * a.slabs * g.C);
        a.ws = static_cast<float*>(g.ws);
        a.sums = a.ws + of_groups;
    } else if (!p.d.resident) {
        const size_t of_groups = 2 * (size_t)g.N * a.slabs * g.groups;
        p.bytes = sizeof(double) * of_groups + sizeof(float) * (size_t)g.N * g.groups;
        a.stats = static_cast<double*>(g.ws);
        a.first = reinterpret_cast<float*>(a.stats + of_groups);
    }
    return p;
}

bool vector_possible(const GroupNormArgs& g) { return gnorm::vector_possible(g.C, g.groups, element_bytes(g.dtype)); }

Plan make_plan(const GroupNormArgs& g, bool backward)
{
    const int V = 16 / element_bytes(g.dtype);
    const bool vector = vector_possible(g) && whole_units(g.x, g.xs, V) && (!g.y || whole_units(g.y, g.ys, V)) && (!backward || whole_units(g.dy, g.dys, V));
    return make_plan_with(g, backward, vector);
}

bool empty(const GroupNormArgs& g) { return g.N == 0 || (int64_t)g.H * g.W == 0; }

hipError_t launch_empty(const GroupNormArgs& g, bool backward, hipStream_t stream)
{
    Args a{};
    a.N = g.N;
    a.C = g.C;
    a.groups = g.groups;
    a.eps = g.eps;
    a.mean = g.mean;
    a.rstd = g.rstd;
    a.dgamma = g.dgamma;
    a.dbeta = g.dbeta;
    a.param_dtype = g.param_dtype;
    const int64_t n = backward ? g.C : (int64_t)g.N * g.groups;
    if (n == 0 || (backward ? !g.dgamma && !g.dbeta : !g.mean && !g.rstd)) return hipSuccess;
    return launch_kernel(empty_kernel, dim3((unsigned)((n + kThreads - 1) / kThreads)), dim3(kThreads), 0, stream, a, backward);
}

// f(V) for the plan's width.
template <typename T, typename F>
hipError_t with_width(const Plan& p, F f)
{
    return p.vector ? f(std::integral_constant<int, 16 / (int)sizeof(T)>{}) : f(std::integral_constant<int, 1>{});
}

}  // namespace

size_t group_norm_workspace_bytes(const GroupNormArgs& g, bool backward)
{
    if (empty(g)) return 0;
    const size_t plain = make_plan_with(g, backward, false).bytes;
    return vector_possible(g) ? std::max(plain, make_plan_with(g, backward, true).bytes) : plain;
}

hipError_t launch_group_norm(const GroupNormArgs& g, hipStream_t stream)
{
    if (empty(g)) return launch_empty(g, false, stream);
    const Plan p = make_plan(g, false);
    const Division& d = p.d;
    const dim3 grid(d.slabs, d.chunks, g.N);
    return with_type(g.dtype, [&](auto t) {
        using T = decltype(t);
        return with_width<T>(p, [&](auto v) {
            constexpr int V = decltype(v)::value;
            if constexpr (V > 1) {
                if (d.resident)
                    return with_activation(g.act, [&](auto act) {
                        constexpr int ACT = decltype(act)::value;
                        auto launch = [&](auto kernel, LdsLimit& limit) {
                            const hipError_t e = d.resident_lds > 65536 ? raise_lds_limit(reinterpret_cast<const void*>(kernel), d.resident_lds, limit) : hipSuccess;
                            return e != hipSuccess ? e : launch_kernel(kernel, grid, dim3(d.resident), d.resident_lds, stream, p.args);
                        };
                        static LdsLimit limits[3];
                        if (d.held == 4) return launch(resident_kernel<T, ACT, 4>, limits[0]);
                        return d.held == 8 ? launch(resident_kernel<T, ACT, 8>, limits[1]) : launch(resident_kernel<T, ACT, 16>, limits[2]);
                    });
            }
            static LdsLimit limit;
            hipError_t e = d.sums_lds > 65536 ? raise_lds_limit(reinterpret_cast<const void*>(stats_kernel<T, V>), d.sums_lds, limit) : hipSuccess;
            if (e == hipSuccess) e = launch_kernel(stats_kernel<T, V>, grid, dim3(kThreads), d.sums_lds, stream, p.args);
            if (e != hipSuccess) return e;
            return with_activation(g.act, [&](auto act) {
                static LdsLimit limit_apply;
                if (d.apply_lds > 65536) {
                    const hipError_t f = raise_lds_limit(reinterpret_cast<const void*>(apply_kernel<T, V, decltype(act)::value>), d.apply_lds, limit_apply);
                    if (f != hipSuccess) return f;
                }
                return launch_kernel(apply_kernel<T, V, decltype(act)::value>, grid, dim3(kThreads), d.apply_lds, stream, p.args);
            });
        });
    });
}

hipError_t launch_group_norm_backward(const GroupNormArgs& g, hipStream_t stream)
{
    if (empty(g)) return launch_empty(g, true, stream);
    const Plan p = make_plan(g, true);
    const Division& d = p.d;
    const dim3 grid(d.slabs, d.chunks, g.N);
    return with_type(g.dtype, [&](auto t) {
        using T = decltype(t);
        return with_width<T>(p, [&](auto v) {
            constexpr int V = decltype(v)::value;
            return with_activation(g.act, [&](auto act) {
                constexpr int ACT = decltype(act)::value;
                static LdsLimit limit, limit_apply;
                if constexpr (V > 1) {
                    if (d.resident) {
                        auto launch = [&](auto kernel, LdsLimit& held) {
                            const hipError_t f = d.resident_lds > 65536 ? raise_lds_limit(reinterpret_cast<const void*>(kernel), d.resident_lds, held) : hipSuccess;
                            return f != hipSuccess ? f : launch_kernel(kernel, grid, dim3(d.resident), d.resident_lds, stream, p.args);
                        };
                        static LdsLimit limits[2];
                        const hipError_t f = d.held == 4 ? launch(backward_resident_kernel<T, ACT, 4>, limits[0]) : launch(backward_resident_kernel<T, ACT, 8>, limits[1]);
                        if (f != hipSuccess || (!g.dgamma && !g.dbeta)) return f;
                        return launch_kernel(backward_parameters_kernel, dim3(1, d.chunks, 1), dim3(kThreads), 0, stream, p.args);
                    }
                }
                hipError_t e = d.sums_lds > 65536 ? raise_lds_limit(reinterpret_cast<const void*>(backward_sums_kernel<T, V, ACT>), d.sums_lds, limit) : hipSuccess;
                if (e == hipSuccess) e = launch_kernel(backward_sums_kernel<T, V, ACT>, grid, dim3(kThreads), d.sums_lds, stream, p.args);
                if (e != hipSuccess) return e;
                if (!g.y) return launch_kernel(backward_parameters_kernel, dim3(1, d.chunks, 1), dim3(kThreads), 0, stream, p.args);
                if (d.apply_lds > 65536) e = raise_lds_limit(reinterpret_cast<const void*>(backward_apply_kernel<T, V, ACT>), d.apply_lds, limit_apply);
                return e != hipSuccess ? e : launch_kernel(backward_apply_kernel<T, V, ACT>, dim3(grid.x, grid.y, grid.z + (g.dgamma || g.dbeta ? 1 : 0)), dim3(kThreads), d.apply_lds, stream, p.args);
            });
        });
    });
}

}  // namespace anr
