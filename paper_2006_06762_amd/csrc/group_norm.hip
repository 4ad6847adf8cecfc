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
    int table;                      // floats of a table of the kernels that read twice
    size_t bytes;                   // of workspace
    size_t lds;                     // of the kernels that sum
    int resident;                   // threads of the resident kernel, or 0
    int held;                       // its vectors a thread: 4, 8 or 16
    size_t resident_lds;
};

constexpr int kResidentThreads = 1024;

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

// Vectors that a thread of a full work-group holds of a chunk, which has at most 256 columns of them.
int held_by(const Args& a)
{
    const int rows = kResidentThreads / (a.chunk / kHeldChannels);
    return (a.HW + rows - 1) / rows;
}

// Where the resident kernels run: a chunk of an image fits the registers of a work-group (vectors of four channels a thread), and all work-groups the
// CUs at once, at 1024 threads each. 256 channels, groups of 8, SiLU, against the kernels that read twice (us, resident / not):
// forward, 16 bits, 20^2 x 16 images (7 vectors) 9.0 / 13.3, 28^2 x 64 (13) 17 / 22; float32 20^2 x 16 (4) 10.8 / 12.3, but 24^2 x 4 (5) 11.3 / 9.7, 28^2 x 1
// (7) 11.8 / 10.2, x 16 15.1 / 14.7, with work-groups for most CUs 28^2 x 24 17.1 / 18.0, 32^2 x 32 20.6 / 24.7, 40^2 x 28 (13) 27.6 / 30.1.
// Backward, float32 28^2 x 1 11.5 / 12.3, x 32 23.0 / 29.5, 24^2 x 4 11.0 / 10.3; 16 bits 20^2 x 16 12.3 / 13.6, x 64 19.8 / 21.6, 28^2 x 16 (13) 22 / 19.
// More than fit at once: float32 20^2 x 40 21.3 / 16.3, 23.1 / 20.3, 10^2 x 128 27.8 / 15.1; bf16 14^2 x 128 16.1 / 17.3, 21.1 / 19.7, 7^2 x 256 22.6 / 16.1
// (512 of 448 threads fit: float32 7^2 x 64 7.5 / 10.4).
bool resident_pays(const GroupNormArgs& g, const Args& a, bool backward, int64_t work_groups)
{
    const int columns = a.chunk / kHeldChannels;
    if (columns > 256) return false;
    const int64_t threads = std::min<int64_t>(kResidentThreads, ((int64_t)a.HW * columns + 63) / 64 * 64);
    if (work_groups * threads > 256 * kResidentThreads) return false;
    return held_by(a) <= (backward ? 8 : g.dtype != ANR_F32 || work_groups >= 192 ? 16 : 4);
}

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

    const int es = element_bytes(g.dtype), V = vector ? 16 / es : 1;
    p.vector = vector;
    // Whole groups and whole units, at least a line of 128 bytes of a pixel.
    const int least = std::min(common_multiple(a.cg, V), g.C);
    auto chunk_of = [&](int bytes) { return std::min(g.C, least * std::max(1, (bytes / es + least - 1) / least)); };
    a.chunk = chunk_of(128);
    p.chunks = (g.C + a.chunk - 1) / a.chunk;
    // Resident kernels take chunks of 64 bytes where work-groups of 128 would be half the CUs or fewer: the backward pass, and the forward one where a thread
    // has more than four vectors. 256 channels, chunks of 128 / 64 bytes (us): backward, float32 14^2 x 16 images 9.9 / 10.0, 20^2 x 1 10.5 / 10.0, 28^2 x 1
    // 14.3 / 11.5, x 16 18.6 / 16.4; bf16 14^2 x 32 11.7 / 10.4, 20^2 x 16 15.5 / 12.4. Forward, bf16 14^2 x 32 8.0 / 8.6, 20^2 x 16 9.7 / 9.0, x 48 (more
    // than half the CUs) 11.1 / 17.2, 28^2 x 16 14.0 / 11.3. Of maps that only the halves hold, those of 16-bit types with 64 work-groups, forward: against the
    // kernels that read twice bf16 36^2 x 16 17.3 / 15.1, but 40^2 x 1 12.2 / 14.0, and backward 28^2 x 16 15.6 / 17.4.
    const int64_t work_groups = (int64_t)p.chunks * g.N;
    if (vector && chunk_of(64) < a.chunk && work_groups <= 128 &&
        (resident_pays(g, a, backward, work_groups) ? backward || held_by(a) > 4 : !backward && g.dtype != ANR_F32 && work_groups >= 64)) {
        Args half = a;
        half.chunk = chunk_of(64);
        if (resident_pays(g, half, backward, work_groups)) {
            a.chunk = half.chunk;
            p.chunks = (g.C + a.chunk - 1) / a.chunk;
            a.halves = true;
        }
    }
    const int line = 128 / es;
    a.streaming = a.chunk % line == 0 && (reinterpret_cast<uintptr_t>(g.y) & 127) == 0 && g.ys[0] % line == 0 && g.ys[1] % line == 0 && g.ys[2] % line == 0;
    const int columns = a.chunk / V, rows = kThreads / std::min(columns, kThreads);
    p.table = table_floats(std::min(a.chunk, kThreads * V));
    // Slabs: about four work-groups per CU as far as each thread has eight pixels (float32: four), one per CU as far as it has two, and at
    // most 128 that are joined. (Eight or four, backward, 320 channels: float32 8 x 56^2 47 / 36 us, bf16 34 / 35, 4 x 95 x 63 32 / 34.)
    const int64_t others = (int64_t)p.chunks * g.N;
    int64_t slabs = std::min((1024 + others - 1) / others, (int64_t)a.HW / ((es == 4 ? 4 : 8) * rows));
    slabs = std::max(slabs, std::min((256 + others - 1) / others, (int64_t)a.HW / (2 * rows)));
    slabs = std::max<int64_t>(1, std::min<int64_t>(slabs, 128));
    // Work-groups go round-robin to the eight XCDs: those that share the lines at a chunk's ends to the same one (4 x 95 x 63 x 320 bf16, chunks of 160 bytes,
    // 29 / 24 slabs, forward 21.7 / 20.4 us, backward 27.8 / 25.3; level where chunks are whole lines).
    if (slabs > 8) slabs = slabs / 8 * 8;
    a.slab_pixels = (int)((a.HW + slabs - 1) / slabs);
    a.slabs = (a.HW + a.slab_pixels - 1) / a.slab_pixels;
    p.lds = sizeof(float) * (2 * (size_t)rows * a.chunk + (backward ? 4 : 1) * (size_t)p.table);
    if (vector && resident_pays(g, a, backward, others)) {
        const int held_columns = a.chunk / kHeldChannels;
        const int64_t vectors = (int64_t)a.HW * held_columns;
        p.resident = (int)std::min<int64_t>(kResidentThreads, (vectors + 63) / 64 * 64);
        p.resident = std::max(p.resident, (held_columns + 63) / 64 * 64);
        const int resident_rows = p.resident / held_columns, each = (a.HW + resident_rows - 1) / resident_rows;
        p.held = each <= 4 ? 4 : each <= 8 ? 8 : 16;
        const size_t groups = a.chunk / a.cg;
        p.resident_lds = sizeof(float) * (backward ? 6 * (size_t)table_floats(a.chunk) + table_floats(2 * groups) + 2 * (size_t)resident_rows * a.chunk + p.resident
                                                   : 3 * (size_t)table_floats(a.chunk) + table_floats(groups) + (size_t)resident_rows * a.chunk);
        a.slabs = 1;
        a.slab_pixels = a.HW;
    }
    const size_t of_groups = p.resident ? 0 : sizeof(float) * 2 * (size_t)g.N * a.slabs * g.groups;
    p.bytes = of_groups + (backward ? sizeof(float) * 2 * (size_t)g.N * a.slabs * g.C : of_groups / (2 * (size_t)a.slabs));
    a.ws = static_cast<float*>(g.ws);
    a.first = a.sums = a.ws + of_groups / sizeof(float);
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
            if constexpr (V > 1) {
                if (p.resident)
                    return with_activation(g.act, [&](auto act) {
                        constexpr int ACT = decltype(act)::value;
                        auto launch = [&](auto kernel, LdsLimit& limit) {
                            const hipError_t e = p.resident_lds > 65536 ? raise_lds_limit(reinterpret_cast<const void*>(kernel), p.resident_lds, limit) : hipSuccess;
                            return e != hipSuccess ? e : launch_kernel(kernel, grid, dim3(p.resident), p.resident_lds, stream, p.args);
                        };
                        static LdsLimit limits[3];
                        if (p.held == 4) return launch(resident_kernel<T, ACT, 4>, limits[0]);
                        return p.held == 8 ? launch(resident_kernel<T, ACT, 8>, limits[1]) : launch(resident_kernel<T, ACT, 16>, limits[2]);
                    });
            }
            static LdsLimit limit;
            hipError_t e = p.lds > 65536 ? raise_lds_limit(reinterpret_cast<const void*>(stats_kernel<T, V>), p.lds, limit) : hipSuccess;
            if (e == hipSuccess) e = launch_kernel(stats_kernel<T, V>, grid, dim3(kThreads), p.lds, stream, p.args);
            if (e != hipSuccess) return e;
            const size_t apply_lds = sizeof(float) * (3 * (size_t)p.table + 2 * (size_t)(p.args.chunk / p.args.cg));
            return with_activation(g.act, [&](auto act) {
                static LdsLimit limit_apply;
                if (apply_lds > 65536) {
                    const hipError_t f = raise_lds_limit(reinterpret_cast<const void*>(apply_kernel<T, V, decltype(act)::value>), apply_lds, limit_apply);
                    if (f != hipSuccess) return f;
                }
                return launch_kernel(apply_kernel<T, V, decltype(act)::value>, grid, dim3(kThreads), apply_lds, stream, p.args);
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
                static LdsLimit limit, limit_apply;
                const size_t apply_lds = sizeof(float) * std::max<size_t>(6 * (size_t)p.table + 2 * (size_t)(p.args.chunk / p.args.cg), kThreads);
                if constexpr (V > 1) {
                    if (p.resident) {
                        auto launch = [&](auto kernel, LdsLimit& held) {
                            const hipError_t f = p.resident_lds > 65536 ? raise_lds_limit(reinterpret_cast<const void*>(kernel), p.resident_lds, held) : hipSuccess;
                            return f != hipSuccess ? f : launch_kernel(kernel, grid, dim3(p.resident), p.resident_lds, stream, p.args);
                        };
                        static LdsLimit limits[2];
                        const hipError_t f = p.held == 4 ? launch(backward_resident_kernel<T, ACT, 4>, limits[0]) : launch(backward_resident_kernel<T, ACT, 8>, limits[1]);
                        if (f != hipSuccess || (!g.dgamma && !g.dbeta)) return f;
                        return launch_kernel(backward_parameters_kernel, dim3(1, p.chunks, 1), dim3(kThreads), 0, stream, p.args);
                    }
                }
                hipError_t e = p.lds > 65536 ? raise_lds_limit(reinterpret_cast<const void*>(backward_sums_kernel<T, V, ACT>), p.lds, limit) : hipSuccess;
                if (e == hipSuccess) e = launch_kernel(backward_sums_kernel<T, V, ACT>, grid, dim3(kThreads), p.lds, stream, p.args);
                if (e != hipSuccess) return e;
                if (!g.y) return launch_kernel(backward_parameters_kernel, dim3(1, p.chunks, 1), dim3(kThreads), 0, stream, p.args);
                if (apply_lds > 65536) e = raise_lds_limit(reinterpret_cast<const void*>(backward_apply_kernel<T, V, ACT>), apply_lds, limit_apply);
                return e != hipSuccess ? e : launch_kernel(backward_apply_kernel<T, V, ACT>, dim3(grid.x, grid.y, grid.z + (g.dgamma || g.dbeta ? 1 : 0)), dim3(kThreads), apply_lds, stream, p.args);
            });
        });
    });
}

}  // namespace anr
