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
    bool vector;                    // 16-byte loads
    int chunks;
    size_t bytes;                   // of workspace
    size_t lds;                     // of the kernels that sum
};

int common_multiple(int a, int b)
{
    int x = a, y = b;
    while (y) {
        const int r = x % y;
        x = y;
        y = r;
    }
    return a / x * b;
}

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

    const int es = element_bytes(g.dtype), V = vector ? 16 / es : 1;
    p.vector = vector;
    // Whole groups and whole units, at least a line of 128 bytes of a pixel.
    const int least = std::min(common_multiple(a.cg, V), g.C);
    a.chunk = std::min(g.C, least * std::max(1, (128 / es + least - 1) / least));
    p.chunks = (g.C + a.chunk - 1) / a.chunk;
    const int columns = a.chunk / V, rows = kThreads / std::min(columns, kThreads);
    // Slabs: about four work-groups per CU, four pixels for each thread or more, and at most 128 that are joined.
    const int64_t others = (int64_t)p.chunks * g.N;
    int64_t slabs = (1024 + others - 1) / others;
    slabs = std::max<int64_t>(1, std::min({slabs, (int64_t)a.HW / (4 * rows), (int64_t)128}));
    a.slab_pixels = (int)((a.HW + slabs - 1) / slabs);
    a.slabs = (a.HW + a.slab_pixels - 1) / a.slab_pixels;
    p.lds = sizeof(float) * 2 * (size_t)std::max(rows, 1) * a.chunk;
    const size_t partial = sizeof(float) * 2 * (size_t)g.N * a.slabs * (backward ? (size_t)g.C : (size_t)g.groups);
    const size_t sums = backward ? sizeof(float) * 2 * (size_t)g.N * g.C : 0;
    p.bytes = partial + sums + (backward ? sizeof(float) * 2 * (size_t)g.N * g.groups : 0);
    a.ws = static_cast<float*>(g.ws);
    a.sums = a.ws + partial / sizeof(float);
    a.group_sums = a.sums + sums / sizeof(float);
    return p;
}

bool vector_possible(const GroupNormArgs& g)
{
    const int V = 16 / element_bytes(g.dtype);
    // (a chunk of whole groups and units is held in LDS)
    return g.C % V == 0 && std::min(common_multiple(g.C / g.groups, V), g.C) <= 8192;
}

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
    const dim3 grid(p.args.slabs, p.chunks, g.N);
    return with_type(g.dtype, [&](auto t) {
        using T = decltype(t);
        return with_width<T>(p, [&](auto v) {
            constexpr int V = decltype(v)::value;
            static LdsLimit limit;
            hipError_t e = p.lds > 65536 ? raise_lds_limit(reinterpret_cast<const void*>(stats_kernel<T, V>), p.lds, limit) : hipSuccess;
            if (e == hipSuccess) e = launch_kernel(stats_kernel<T, V>, grid, dim3(kThreads), p.lds, stream, p.args);
            if (e != hipSuccess) return e;
            return with_activation(g.act, [&](auto act) {
                return launch_kernel(apply_kernel<T, V, decltype(act)::value>, grid, dim3(kThreads), sizeof(float) * 2 * (p.args.chunk / p.args.cg), stream, p.args);
            });
        });
    });
}

hipError_t launch_group_norm_backward(const GroupNormArgs& g, hipStream_t stream)
{
    if (empty(g)) return launch_empty(g, true, stream);
    const Plan p = make_plan(g, true);
    const dim3 grid(p.args.slabs, p.chunks, g.N);
    return with_type(g.dtype, [&](auto t) {
        using T = decltype(t);
        return with_width<T>(p, [&](auto v) {
            constexpr int V = decltype(v)::value;
            return with_activation(g.act, [&](auto act) {
                constexpr int ACT = decltype(act)::value;
                static LdsLimit limit, limit_groups;
                const size_t lds = sizeof(float) * 2 * p.args.chunk;
                hipError_t e = p.lds > 65536 ? raise_lds_limit(reinterpret_cast<const void*>(backward_sums_kernel<T, V, ACT>), p.lds, limit) : hipSuccess;
                if (e == hipSuccess && lds > 65536) e = raise_lds_limit(reinterpret_cast<const void*>(backward_groups_kernel), lds, limit_groups);
                if (e == hipSuccess) e = launch_kernel(backward_sums_kernel<T, V, ACT>, grid, dim3(kThreads), p.lds, stream, p.args);
                if (e == hipSuccess) e = launch_kernel(backward_groups_kernel, dim3(1, p.chunks, g.N), dim3(kThreads), lds, stream, p.args);
                if (e != hipSuccess) return e;
                if (!g.y) return launch_kernel(backward_parameters_kernel, dim3(1, p.chunks, 1), dim3(kThreads), 0, stream, p.args);
                return launch_kernel(backward_apply_kernel<T, V, ACT>, grid, dim3(kThreads), 0, stream, p.args);
            });
        });
    });
}

}  // namespace anr
