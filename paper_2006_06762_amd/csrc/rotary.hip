// Rotary positions with several axes: pairs (u, v) of a token's dimensions become (u cos - v sin, u sin + v cos), with the
// angle positions[axis of the pair] * inv_freq[pair].
//
// Bound: by memory, each element is read and written once.  The angle of a pair is the same for all heads, so a thread
// takes one column (V pairs, or V dimensions that are only copied) of one token and turns it in several heads with one
// sine and cosine: it is computed once per column and head group.  Far positions need more than 32 bits of
// the angle (a position of 10^6 at frequency 1 leaves 0.06 of a radian in a float), so it is formed in 64 bits as quarter
// turns and reduced there to an eighth of a turn on either side, |t| <= pi/4, where the Taylor polynomials of degree 9 and 10
// are off by t^11 / 11! < 2e-9 and t^12 / 12! < 2e-10 of 1: below half a unit of float's last place, 3e-8.
#include "blocks_internal.h"
#include "element_types.h"

#include <algorithm>

namespace anr {
namespace {

constexpr int kThreads = 256;

struct RotaryKernelArgs {
    const void *q, *k;
    void *q_out, *k_out;
    const void* positions;
    const float* inv_freq;
    int64_t qs[3], ks[3], qos[3], kos[3], ps[3];
    int S, H, heads;                // heads: of q and k
    int section_end[4];             // first pair behind each axis
    int pairs, pairing, inverse, pos_type;
    int pair_columns, columns;      // columns of V pairs; with those of V dimensions that are copied
    int rest;                       // first dimension that is copied
    int head_groups;                // threads that share a token's column
    uint32_t items;
    FastDiv by_columns, by_groups, by_s;
};

__device__ __forceinline__ double position(const void* p, int64_t i, int type)
{
    return type == ANR_POS_I64 ? (double)static_cast<const int64_t*>(p)[i] : type == ANR_POS_I32 ? (double)static_cast<const int32_t*>(p)[i] : (double)static_cast<const float*>(p)[i];
}

// cos and sin of position * frequency.
__device__ __forceinline__ void turn_of(double pos, float freq, float& c, float& s)
{
    const double quarters = pos * (double)freq * 0.63661977236758134308;       // 2 / pi
    const double whole = rint(quarters);
    const float t = (float)(quarters - whole) * 1.57079632679489662f, t2 = t * t;
    const float sine = fmaf(t * t2, fmaf(t2, fmaf(t2, fmaf(t2, 1.f / 362880.f, -1.f / 5040.f), 1.f / 120.f), -1.f / 6.f), t);
    const float cosine = fmaf(t2, fmaf(t2, fmaf(t2, fmaf(t2, fmaf(t2, -1.f / 3628800.f, 1.f / 40320.f), -1.f / 720.f), 1.f / 24.f), -0.5f), 1.f);
    const int quadrant = (int)(whole - 4.0 * floor(0.25 * whole));             // 0 .. 3 (an infinite or NaN position: any)
    const float a = quadrant & 1 ? sine : cosine, b = quadrant & 1 ? cosine : sine;
    c = quadrant == 1 || quadrant == 2 ? -a : a;
    s = quadrant & 2 ? -b : b;
}

// ADJACENT: the V pairs of a column are 2 V dimensions in a row, else two runs of V.
template <typename T, int V, bool ADJACENT>
__global__ __launch_bounds__(kThreads) void rotary_kernel(const RotaryKernelArgs a)
{
    const uint32_t item = blockIdx.x * kThreads + threadIdx.x;           // (below 2^31: see the launch)
    if (item >= a.items) return;
    const int token_group = a.by_columns.div((int)item), col = (int)item - token_group * a.columns;
    const int token = a.by_groups.div(token_group), group = token_group - token * a.head_groups;
    const int b = a.by_s.div(token), s = token - b * a.S;
    const int64_t in_q = b * a.qs[0] + s * a.qs[1], in_k = b * a.ks[0] + s * a.ks[1];
    const int64_t out_q = b * a.qos[0] + s * a.qos[1], out_k = b * a.kos[0] + s * a.kos[1];
    auto source = [&](int h) { return h < a.H ? static_cast<const T*>(a.q) + in_q + h * a.qs[2] : static_cast<const T*>(a.k) + in_k + (h - a.H) * a.ks[2]; };
    auto target = [&](int h) { return h < a.H ? static_cast<T*>(a.q_out) + out_q + h * a.qos[2] : static_cast<T*>(a.k_out) + out_k + (h - a.H) * a.kos[2]; };
    if (col >= a.pair_columns) {
        constexpr int W = ADJACENT && V > 1 ? 2 * V : V;
        const int d = a.rest + (col - a.pair_columns) * W;
        for (int h = group; h < a.heads; h += a.head_groups) *reinterpret_cast<Pack<T, W>*>(target(h) + d) = *reinterpret_cast<const Pack<T, W>*>(source(h) + d);
        return;
    }
    const int pair = col * V;
    // (the pairs of a column lie in one section where sections have blocks of their own; else each has its axis)
    int axis0 = 0;
#pragma unroll
    for (int i = 0; i < 3; ++i) axis0 += pair >= a.section_end[i];
    int first = pair, second = a.pairs + pair;
    if (a.pairing == ANR_ROTARY_SECTION_HALVES) {
        const int begin = axis0 ? a.section_end[axis0 - 1] : 0, length = a.section_end[axis0] - begin;
        first = begin + pair;                       // 2 begin + (pair - begin)
        second = first + length;
    }
    // the elements of HEADS heads are on their way while the angles are formed, and those of the next ones while these are turned
    constexpr int HEADS = 4;
    Pack<T, 2 * V> x[HEADS];
    auto load = [&](int h0) {
#pragma unroll
        for (int j = 0; j < HEADS; ++j) {
            const T* const from = source(min(h0 + j * a.head_groups, a.heads - 1));
            if (ADJACENT && V > 1) {
                x[j] = *reinterpret_cast<const Pack<T, 2 * V>*>(from + 2 * pair);
            } else {
                const Pack<T, V> lo = *reinterpret_cast<const Pack<T, V>*>(from + (ADJACENT ? 2 * pair : first)), hi = *reinterpret_cast<const Pack<T, V>*>(from + (ADJACENT ? 2 * pair + 1 : second));
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    x[j].v[i] = lo.v[i];
                    x[j].v[V + i] = hi.v[i];
                }
            }
        }
    };
    load(group);
    __builtin_amdgcn_sched_barrier(0);
    float c[V], sn[V];
#pragma unroll
    for (int i = 0; i < V; ++i) {
        int axis = 0;
#pragma unroll
        for (int j = 0; j < 3; ++j) axis += pair + i >= a.section_end[j];
        const double pos = position(a.positions, axis * a.ps[0] + b * a.ps[1] + s * a.ps[2], a.pos_type);
        turn_of(pos, a.inv_freq[pair + i], c[i], sn[i]);
        sn[i] = a.inverse ? -sn[i] : sn[i];
    }
    for (int h0 = group; h0 < a.heads; h0 += HEADS * a.head_groups) {
        if (h0 != group) load(h0);
#pragma unroll
        for (int j = 0; j < HEADS; ++j) {
            const int h = h0 + j * a.head_groups;
            if (h >= a.heads) continue;
            T* const to = target(h);
            float y[2 * V];
#pragma unroll
            for (int i = 0; i < V; ++i) {
                constexpr int STEP = ADJACENT ? 2 : 1, OTHER = ADJACENT ? 1 : V;
                const float u = to_float(x[j].v[STEP * i]), v = to_float(x[j].v[STEP * i + OTHER]);
                y[STEP * i] = u * c[i] - v * sn[i];
                y[STEP * i + OTHER] = u * sn[i] + v * c[i];
            }
            if (ADJACENT && V > 1) {
                store_floats<T, 2 * V>(to + 2 * pair, y);
            } else {
                float lo[V], hi[V];
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    lo[i] = y[i];
                    hi[i] = y[V + i];
                }
                store_floats<T, V>(to + (ADJACENT ? 2 * pair : first), lo);
                store_floats<T, V>(to + (ADJACENT ? 2 * pair + 1 : second), hi);
            }
        }
    }
}

}  // namespace

hipError_t launch_rotary(const RotaryArgs& g, hipStream_t stream)
{
    const anr_rotary_desc& d = g.d;
    const int64_t tokens = (int64_t)d.B * d.S;
    const int heads = d.H + d.Hk;
    if (tokens == 0 || heads == 0 || d.D == 0) return hipSuccess;
    RotaryKernelArgs a{};
    a.q = g.q;
    a.k = g.k;
    a.q_out = g.q_out;
    a.k_out = g.k_out;
    a.positions = g.positions;
    a.inv_freq = g.inv_freq;
    for (int i = 0; i < 3; ++i) {
        a.qs[i] = d.q_stride[i];
        a.ks[i] = d.k_stride[i];
        a.qos[i] = d.q_out_stride[i];
        a.kos[i] = d.k_out_stride[i];
        a.ps[i] = d.pos_stride[i];
    }
    a.S = d.S;
    a.H = d.H;
    a.heads = heads;
    for (int i = 0; i < 4; ++i) {
        if (i < d.axes) a.pairs += d.section[i];
        a.section_end[i] = a.pairs;
    }
    a.pairing = d.pairing;
    a.inverse = d.inverse;
    a.pos_type = d.pos_type;
    a.rest = 2 * a.pairs;
    const bool adjacent = d.pairing == ANR_ROTARY_ADJACENT;
    return with_type(d.dtype, [&](auto t) {
        using T = decltype(t);
        constexpr int UNIT = 16 / (int)sizeof(T);
        // 16-byte loads where every run of a column starts at a multiple of 16 bytes
        bool whole = d.D % UNIT == 0 && a.rest % UNIT == 0;
        if (d.pairing == ANR_ROTARY_HALVES) whole = whole && a.pairs % UNIT == 0;
        if (d.pairing == ANR_ROTARY_SECTION_HALVES)
            for (int i = 0; i < d.axes; ++i) whole = whole && d.section[i] % UNIT == 0;
        auto aligned = [&](const void* p, const int64_t* s) { return is_aligned16(p) && s[0] % UNIT == 0 && s[1] % UNIT == 0 && s[2] % UNIT == 0; };
        whole = whole && aligned(g.q, a.qs) && aligned(g.q_out, a.qos) && (d.Hk == 0 || (aligned(g.k, a.ks) && aligned(g.k_out, a.kos)));
        auto launch = [&](auto kernel, int pairs_per_column, int copied) {
            RotaryKernelArgs b = a;
            b.pair_columns = a.pairs / pairs_per_column;
            b.columns = b.pair_columns + (d.D - a.rest) / copied;
            // A token's heads are shared by as many threads as fill the card, but a column's angles are worth four heads
            const int64_t per_head = tokens * b.columns;
            b.head_groups = (int)std::min({(int64_t)heads, std::max<int64_t>((heads + 3) / 4, (256 * 1024 + per_head - 1) / per_head), (int64_t)0x7fffff00 / per_head});
            b.items = (uint32_t)(per_head * b.head_groups);
            b.by_columns = make_fastdiv(b.columns);
            b.by_groups = make_fastdiv(b.head_groups);
            b.by_s = make_fastdiv(d.S);
            return launch_kernel(kernel, dim3((unsigned)((b.items + kThreads - 1) / kThreads)), dim3(kThreads), 0, stream, b);
        };
        if (!whole) return adjacent ? launch(rotary_kernel<T, 1, true>, 1, 1) : launch(rotary_kernel<T, 1, false>, 1, 1);
        return adjacent ? launch(rotary_kernel<T, UNIT / 2, true>, UNIT / 2, UNIT) : launch(rotary_kernel<T, UNIT, false>, UNIT, UNIT);
    });
}

}  // namespace anr
