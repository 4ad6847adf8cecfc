// What the group norm's kernels (group_norm_kernel.h) divide and lay out how: plain arithmetic without a device in it, so that a CPU program
// can hold what a launch asks for against what its work-groups use.
#pragma once
#include <stddef.h>
#include <stdint.h>

#include <algorithm>

namespace anr {
namespace gnorm {

constexpr int kThreads = 256;                // of the kernels that read twice
constexpr int kResidentThreads = 1024;
constexpr int kHeldChannels = 4;             // of a vector of the resident kernels (of eight, the constants of 16-bit types' channels left no registers for the data)

// Floats of a table in LDS: whole 16-byte units.
constexpr int table_floats(int channels) { return (channels + 3) & ~3; }

// Threads of a work-group on `channels` channels: columns of V of them by rows of pixels.  A chunk of fewer channels has more rows, and rows x
// channels may be more than a wider one's: 100 channels of 256 threads are 2 rows, 60 are 4.
constexpr int columns_of(int channels, int V) { return channels / V; }
constexpr int rows_of(int channels, int V, int threads) { return threads / (columns_of(channels, V) < threads ? columns_of(channels, V) : threads); }

// Channels that the tables of the kernels that read twice hold at a time.
constexpr int table_channels(int channels, int V) { return channels < kThreads * V ? channels : kThreads * V; }

// Floats of LDS that a work-group on `channels` channels uses: of the kernels that sum (a table and two numbers of 64 bits a channel and row; backward four
// tables), of the resident ones, of those that apply.
constexpr size_t sums_lds_floats(bool backward, int channels, int V)
{
    return (backward ? 4 : 1) * (size_t)table_floats(table_channels(channels, V)) + 4 * (size_t)rows_of(channels, V, kThreads) * channels;
}
constexpr size_t resident_lds_floats(bool backward, int channels, int cg, int threads)
{
    const size_t groups = channels / cg, part = (size_t)rows_of(channels, kHeldChannels, threads) * channels;
    return backward ? 6 * (size_t)table_floats(channels) + table_floats(2 * groups) + 2 * part + 2 * (size_t)threads : 2 * (size_t)table_floats(channels) + 2 * ((size_t)table_floats(groups) + part);
}
constexpr size_t apply_lds_floats(bool backward, int channels, int cg, int V)
{
    const size_t floats = (backward ? 6 : 3) * (size_t)table_floats(table_channels(channels, V)) + (backward ? 2 : 3) * (size_t)(channels / cg);
    return backward && floats < (size_t)2 * kThreads ? (size_t)2 * kThreads : floats;        // (the parameters' gradients take 64 bits a thread)
}

// A call, and how its kernels divide it.
struct Shape {
    int N, HW, C, groups;
    int es;                         // bytes of an element
    bool vector;                    // loads of 16 bytes, else of single elements
    bool backward;
};
struct Division {
    int V;                          // channels of a thread of the kernels that read twice
    int chunk, chunks;              // channels of a chunk, whole groups; the last may have fewer
    bool halves;                    // resident: a chunk's pixel is half a line
    int slabs, slab_pixels;
    int resident;                   // threads of the resident kernel, or 0
    int held;                       // its vectors a thread: 4, 8 or 16
    size_t sums_lds, apply_lds, resident_lds;    // bytes a launch asks for
};

inline int common_multiple(int a, int b)
{
    int x = a, y = b;
    while (y) {
        const int r = x % y;
        x = y;
        y = r;
    }
    return a / x * b;
}

// Whether loads of 16 bytes can be: whole units of a pixel, and a chunk of whole groups and units that LDS holds.
inline bool vector_possible(int C, int groups, int es)
{
    const int V = 16 / es;
    return C % V == 0 && std::min(common_multiple(C / groups, V), C) <= 8192;
}

// Vectors that a thread of a full work-group holds of a chunk, which has at most 256 columns of them.
inline int held_by(const Shape& s, int chunk)
{
    const int rows = rows_of(chunk, kHeldChannels, kResidentThreads);
    return (s.HW + rows - 1) / rows;
}

// Where the resident kernels run: a chunk of an image fits the registers of a work-group (vectors of four channels a thread), and all work-groups the
// CUs at once, at 1024 threads each. 256 channels, groups of 8, SiLU, against the kernels that read twice (us, resident / not):
// forward, 16 bits, 20^2 x 16 images (7 vectors) 7.7 / 11.4, 28^2 x 64 (13) 17.0 / 19.8; float32 20^2 x 16 (4) 8.9 / 10.8, with work-groups for half the CUs
// 24^2 x 16 (5) 9.8 / 11.7, 28^2 x 16 11.7 / 13.1, 40^2 x 16 (13) 17.1 / 18.6, 40^2 x 28 26.4 / 28.9, but for fewer 24^2 x 4 8.3 / 8.6, 28^2 x 1 (7) 8.9 / 9.3, 32^2
// x 4 (8) 9.9 / 9.1, 40^2 x 8 14.3 / 13.3, x 1 12.1 / 8.6.
// Backward, float32 28^2 x 1 11.4 / 10.9, x 32 23.3 / 29.1, 24^2 x 4 10.9 / 10.2, 32^2 x 4 12.9 / 11.3; 16 bits 20^2 x 16 12.7 / 12.4, x 64 20.1 / 23.5, 14^2 x 32 10.6 / 12.0.
// More than fit at once, forward and backward: float32 20^2 x 40 17.3 / 14.3, 23.5 / 20.4, 10^2 x 128 21.3 / 13.4, 26.5 / 17.3; bf16 14^2 x 128 13.8 / 15.0, 23.7 /
// 19.4, 7^2 x 256 19.7 / 14.2, 28.7 / 19.7 (512 of 448 threads fit: float32 7^2 x 64 6.4 / 9.0, 8.9 / 10.3).
inline bool resident_pays(const Shape& s, int chunk, int64_t work_groups)
{
    const int columns = columns_of(chunk, kHeldChannels);
    if (columns > 256) return false;
    const int64_t threads = std::min<int64_t>(kResidentThreads, ((int64_t)s.HW * columns + 63) / 64 * 64);
    if (work_groups * threads > 256 * kResidentThreads) return false;
    return held_by(s, chunk) <= (s.backward ? 8 : s.es == 2 || work_groups >= 128 ? 16 : 4);
}

// f(channels) of the larger of a full chunk and the last one.
template <typename F>
size_t of_chunks(const Division& d, int C, F f)
{
    const int last = C - (d.chunks - 1) * d.chunk;
    return std::max<size_t>(f(d.chunk), f(last));
}

inline Division divide(const Shape& s)
{
    Division d{};
    d.V = s.vector ? 16 / s.es : 1;
    const int cg = s.C / s.groups;
    // Whole groups and whole units, at least a line of 128 bytes of a pixel.
    const int least = std::min(common_multiple(cg, d.V), s.C);
    auto chunk_of = [&](int bytes) { return std::min(s.C, least * std::max(1, (bytes / s.es + least - 1) / least)); };
    auto take = [&](int chunk) {
        d.chunk = chunk;
        d.chunks = (s.C + chunk - 1) / chunk;
    };
    take(chunk_of(128));
    // Resident kernels take chunks of 64 bytes where work-groups of 128 would be half the CUs or fewer: the backward pass, and the forward one where a thread
    // has more than four vectors. 256 channels, chunks of 128 / 64 bytes (us): backward, float32 14^2 x 16 images 10.0 / 9.8, 20^2 x 1 10.7 / 9.9, 28^2 x 1
    // 14.6 / 11.4, x 16 18.9 / 16.4; bf16 14^2 x 32 11.8 / 10.6, 20^2 x 16 15.9 / 12.7. Forward, bf16 14^2 x 32 (4 vectors) 7.0 / 7.0, 20^2 x 16 9.1 / 7.6, x 48 (more
    // than half the CUs) 10.2 / 14.1, 28^2 x 16 14.1 / 9.7. Of maps that only the halves hold, those of 16-bit types with 64 work-groups, forward: against the
    // kernels that read twice bf16 36^2 x 16 14.4 / 15.4, but 40^2 x 1 13.6 / 10.1, float32 52^2 x 8 17.5 / 17.2.
    const int64_t work_groups = (int64_t)d.chunks * s.N;
    if (s.vector && chunk_of(64) < d.chunk && work_groups <= 128 &&
        (resident_pays(s, d.chunk, work_groups) ? s.backward || held_by(s, d.chunk) > 4 : !s.backward && s.es == 2 && work_groups >= 64) &&
        resident_pays(s, chunk_of(64), work_groups)) {
        take(chunk_of(64));
        d.halves = true;
    }
    const int rows = rows_of(d.chunk, d.V, kThreads);
    // Slabs: about four work-groups per CU as far as each thread has eight pixels (float32: four), one per CU as far as it has two, and at
    // most 128 that are joined, 256 where those are less than two work-groups per CU: one map of 1024^2, forward and backward, 128 / 256 slabs, 64 channels bf16
    // 215 / 125 us, 367 / 215, float32 211 / 170, 450 / 291, 256^2 x 64 bf16 24.5 / 24.2, 29.5 / 24.6, but two maps of 256^2 x 64 float32 (four work-groups a slab) 26.9 /
    // 29.8, 36.8 / 46.5. (Eight or four, backward, 320 channels: bf16 8 x 64^2 27.8 / 35.8 us, 4 x 95 x 63 22.6 / 25.9.)
    const int64_t others = (int64_t)d.chunks * s.N;
    int64_t slabs = std::min((1024 + others - 1) / others, (int64_t)s.HW / ((s.es == 4 ? 4 : 8) * rows));
    slabs = std::max(slabs, std::min((256 + others - 1) / others, (int64_t)s.HW / (2 * rows)));
    const int64_t most = others <= 2 ? 256 : 128;
    slabs = std::max<int64_t>(1, std::min(slabs, most));
    // Work-groups go round-robin to the eight XCDs: those that share the lines at a chunk's ends to the same one, so slabs come in eights, next below or above by the
    // pixels that the fullest CU then has: a work-group's start and joins count as two a thread, a second one on the CU adds 0.7 of the first one's time. Below / above, bf16: 4 x 95 x 63 x 320 (29 slabs, 384 / 512
    // work-groups) forward 18.3 / 17.6 us, backward 25.2 / 22.6, 8 x 56^2 x 320 (15, 256 / 512) 21.2 / 18.9, 30.5 / 22.9; float16 13 x 52 x 33 x 48 (20, 208 / 312)
    // backward 12.5 / 16.0, 13 x 123 x 38 x 80 (23, 208 / 312) 23.7 / 26.7. Level where chunks are whole lines.
    if (slabs > 8) {
        auto fullest = [&](int64_t n) { return (0.3 + 0.7 * (double)((n * others + 255) / 256)) * (double)((s.HW + n - 1) / n + 2 * rows); };
        const int64_t below = slabs / 8 * 8, above = std::min(below + 8, most);
        slabs = slabs > below && above <= s.HW / (2 * rows) && fullest(above) < fullest(below) ? above : below;
    }
    d.slab_pixels = (int)((s.HW + slabs - 1) / slabs);
    d.slabs = (s.HW + d.slab_pixels - 1) / d.slab_pixels;
    d.sums_lds = sizeof(float) * of_chunks(d, s.C, [&](int channels) { return sums_lds_floats(s.backward, channels, d.V); });
    d.apply_lds = sizeof(float) * of_chunks(d, s.C, [&](int channels) { return apply_lds_floats(s.backward, channels, cg, d.V); });
    if (s.vector && resident_pays(s, d.chunk, others)) {
        const int columns = columns_of(d.chunk, kHeldChannels);
        const int64_t vectors = (int64_t)s.HW * columns;
        d.resident = (int)std::min<int64_t>(kResidentThreads, (vectors + 63) / 64 * 64);
        d.resident = std::max(d.resident, (columns + 63) / 64 * 64);
        const int resident_rows = rows_of(d.chunk, kHeldChannels, d.resident), each = (s.HW + resident_rows - 1) / resident_rows;
        d.held = each <= 4 ? 4 : each <= 8 ? 8 : 16;
        d.resident_lds = sizeof(float) * of_chunks(d, s.C, [&](int channels) { return resident_lds_floats(s.backward, channels, cg, d.resident); });
        d.slabs = 1;
        d.slab_pixels = s.HW;
    }
    return d;
}

}  // namespace gnorm
}  // namespace anr
