// Rotary positions with several axes: pairs (u, v) of a token's dimensions become (u cos - v sin, u sin + v cos), with the
// angle positions[axis of the pair] * inv_freq[pair].
//
// Bound: by memory, each element is read and written once.  The angle of a pair is the same for all heads: a work-group forms
// those of its tokens once, in LDS, and then turns the tokens' heads, whose first elements are on their way meanwhile.  (With the
// angles formed by each thread for its own column, once for four heads, 786 MB took 260 us.)  Far positions need more than 32 bits of
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
    int tokens, S, H, heads;        // tokens: of all sequences; heads: of q and k
    int section_end[4];             // first pair behind each axis
    int pairs, pairing, inverse, pos_type;
    int pair_columns, columns;      // columns of V pairs; with those of V dimensions (adjacent: of 2 V) that are copied
    int rest;                       // first dimension that is copied
    int group_tokens, group_heads;  // of a work-group
    FastDiv by_columns, by_heads, by_s, by_pairs;
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
// STREAMING: stores go past L2.
template <typename T, int V, bool ADJACENT, bool STREAMING>
__global__ __launch_bounds__(kThreads) void rotary_kernel(const RotaryKernelArgs a)
{
    extern __shared__ __attribute__((aligned(16))) float lds[];      // cosines of [tokens][pairs], then the sines
    constexpr int W = ADJACENT && V > 1 ? 2 * V : V;                 // dimensions of a copied column
    constexpr int AHEAD = 4;                                         // items of a thread that are on their way together
    const int token0 = blockIdx.x * a.group_tokens, tokens = min(a.group_tokens, a.tokens - token0);
    const int head0 = blockIdx.y * a.group_heads, heads = min(a.group_heads, a.heads - head0);
    const int items = tokens * heads * a.columns;
    const float *const cosines = lds, *const sines = lds + a.group_tokens * a.pairs;

    // an item: a column of a head of a token, in the order of packed memory
    struct Item {
        int64_t from, to;           // first element of the head
        bool in_k, copied;
        int first, second, angle;   // dimensions, and where its angles start
    };
    auto item = [&](int i) {
        Item r;
        const int row = a.by_columns.div(i), col = i - row * a.columns;
        const int token = heads == a.group_heads ? a.by_heads.div(row) : row / heads, h = head0 + row - token * heads;
        const int b = a.by_s.div(token0 + token), s = token0 + token - b * a.S;
        r.in_k = h >= a.H;
        const int own = r.in_k ? h - a.H : h;
        r.from = r.in_k ? b * a.ks[0] + s * a.ks[1] + own * a.ks[2] : b * a.qs[0] + s * a.qs[1] + own * a.qs[2];
        r.to = r.in_k ? b * a.kos[0] + s * a.kos[1] + own * a.kos[2] : b * a.qos[0] + s * a.qos[1] + own * a.qos[2];
        r.copied = col >= a.pair_columns;
        const int pair = col * V;
        r.angle = token * a.pairs + pair;
        r.first = ADJACENT ? 2 * pair : pair;
        r.second = ADJACENT ? r.first + V : a.pairs + pair;
        if (a.pairing == ANR_ROTARY_SECTION_HALVES) {
            int axis = 0;
#pragma unroll
            for (int j = 0; j < 3; ++j) axis += pair >= a.section_end[j];
            const int begin = axis ? a.section_end[axis - 1] : 0;
            r.first = begin + pair;                 // 2 begin + (pair - begin)
            r.second = r.first + a.section_end[axis] - begin;
        }
        if (r.copied) {
            r.first = a.rest + (col - a.pair_columns) * W;
            r.second = W > V ? r.first + V : r.first;
        }
        return r;
    };
    Pack<T, 2 * V> x[AHEAD];
    Item at[AHEAD];
    auto load = [&](int i0) {
#pragma unroll
        for (int j = 0; j < AHEAD; ++j) {
            at[j] = item(min(i0 + j * kThreads, items - 1));
            const T* const from = static_cast<const T*>(at[j].in_k ? a.k : a.q) + at[j].from;
            if (ADJACENT && V > 1) {
                x[j] = *reinterpret_cast<const Pack<T, 2 * V>*>(from + at[j].first);
            } else {
                const Pack<T, V> lo = *reinterpret_cast<const Pack<T, V>*>(from + at[j].first), hi = *reinterpret_cast<const Pack<T, V>*>(from + at[j].second);
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    x[j].v[i] = lo.v[i];
                    x[j].v[V + i] = hi.v[i];
                }
            }
        }
    };
    load(threadIdx.x);
    for (int e = threadIdx.x; e < tokens * a.pairs; e += kThreads) {
        const int token = a.by_pairs.div(e), pair = e - token * a.pairs;
        const int b = a.by_s.div(token0 + token), s = token0 + token - b * a.S;
        int axis = 0;
#pragma unroll
        for (int j = 0; j < 3; ++j) axis += pair >= a.section_end[j];
        float c, sn;
        turn_of(position(a.positions, axis * a.ps[0] + b * a.ps[1] + s * a.ps[2], a.pos_type), a.inv_freq[pair], c, sn);
        lds[e] = c;
        lds[a.group_tokens * a.pairs + e] = a.inverse ? -sn : sn;
    }
    __syncthreads();
    for (int i0 = threadIdx.x; i0 < items; i0 += AHEAD * kThreads) {
        if (i0 >= AHEAD * kThreads) load(i0);
#pragma unroll
        for (int j = 0; j < AHEAD; ++j) {
            if (i0 + j * kThreads >= items) continue;
            T* const to = static_cast<T*>(at[j].in_k ? a.k_out : a.q_out) + at[j].to;
            Pack<T, 2 * V> out = x[j];
            if (!at[j].copied) {
                float y[2 * V];
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    constexpr int STEP = ADJACENT ? 2 : 1, OTHER = ADJACENT ? 1 : V;
                    const float c = cosines[at[j].angle + i], sn = sines[at[j].angle + i];
                    const float u = to_float(x[j].v[STEP * i]), v = to_float(x[j].v[STEP * i + OTHER]);
                    y[STEP * i] = u * c - v * sn;
                    y[STEP * i + OTHER] = u * sn + v * c;
                }
                out = pack_floats<T, 2 * V>(y);
            }
            if (ADJACENT && V > 1) {
                store_pack<STREAMING>(to + at[j].first, out);
            } else {
                Pack<T, V> lo, hi;
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    lo.v[i] = out.v[i];
                    hi.v[i] = out.v[V + i];
                }
                store_pack<STREAMING>(to + at[j].first, lo);
                if (!at[j].copied) store_pack<STREAMING>(to + at[j].second, hi);
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
        // Stores past L2 where they cover runs of 64 bytes: 33 k tokens of 16 heads, past L2 / not, TB/s: float32 halves of 64 pairs 6.4 / 4.9, of 32 6.2 /
        // 5.6, of 16 4.9 / 5.6, bf16 of 64 6.1 / 5.5, of 32 4.9 / 5.1, of 16 3.1 / 4.1; adjacent 36 4.9 / 4.3; 8 k tokens of 8 heads, float32 of 16 4.4 / 3.7.
        // With the scores that read them next, float32, q and k of 12 heads of 64: 128 tokens 8.5 / 8.3 us, 16 x 128 13.4 / 14.2, 512 11.7 / 12.2.
        constexpr int LINE = 64 / (int)sizeof(T);
        bool streaming = adjacent || (d.pairing == ANR_ROTARY_HALVES && a.pairs % LINE == 0);
        if (d.pairing == ANR_ROTARY_SECTION_HALVES) {
            streaming = true;
            for (int i = 0; i < d.axes; ++i) streaming = streaming && d.section[i] % LINE == 0;
        }
        auto launch = [&](auto kernel, int pairs_per_column, int copied) {
            RotaryKernelArgs b = a;
            b.tokens = (int)tokens;
            b.pair_columns = a.pairs / pairs_per_column;
            b.columns = b.pair_columns + (d.D - a.rest) / copied;
            // A work-group has the angles of 512 pairs at most (1024 of one token) and eight items a thread; few tokens share their heads among
            // work-groups as far as there are CUs for them, with an item a thread or more
            const int64_t of_token = (int64_t)heads * b.columns;
            b.group_tokens = (int)std::max<int64_t>(1, std::min({(int64_t)512 / std::max(1, a.pairs), 8 * kThreads / of_token, tokens}));
            while (b.group_tokens > 1 && (tokens + b.group_tokens - 1) / b.group_tokens < 1024) b.group_tokens = (b.group_tokens + 1) / 2;
            const int64_t blocks = (tokens + b.group_tokens - 1) / b.group_tokens, items = b.group_tokens * of_token;
            const int64_t shares = std::max<int64_t>((items + 16 * kThreads - 1) / (16 * kThreads), std::min<int64_t>(512 / blocks, items / kThreads));
            b.group_heads = (int)std::max<int64_t>(1, heads / std::max<int64_t>(1, shares));
            b.by_columns = make_fastdiv(b.columns);
            b.by_heads = make_fastdiv(b.group_heads);
            b.by_s = make_fastdiv(d.S);
            b.by_pairs = make_fastdiv(std::max(1, a.pairs));
            return launch_kernel(kernel, dim3((unsigned)blocks, (unsigned)((heads + b.group_heads - 1) / b.group_heads)), dim3(kThreads),
                                 sizeof(float) * 2 * (size_t)b.group_tokens * a.pairs, stream, b);
        };
        if (!whole) return adjacent ? launch(rotary_kernel<T, 1, true, false>, 1, 1) : launch(rotary_kernel<T, 1, false, false>, 1, 1);
        if (adjacent) return launch(rotary_kernel<T, UNIT / 2, true, true>, UNIT / 2, UNIT);
        return streaming ? launch(rotary_kernel<T, UNIT, false, true>, UNIT, UNIT) : launch(rotary_kernel<T, UNIT, false, false>, UNIT, UNIT);
    });
}

}  // namespace anr
