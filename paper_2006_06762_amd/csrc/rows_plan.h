// How rows of C values are dealt to waves (rows_device.h): plain arithmetic without a device in it.
#pragma once
#include <stdint.h>

namespace anr {
namespace rows {

struct Plan {
    int units;                      // of a thread: a power of two
    int threads;                    // of a row: 8, 16 or 32, or whole waves
    int rows;                       // of a work-group
};

constexpr int kHeld = 32;           // floats of a thread in work-groups of up to 1024 threads
constexpr int kHeldBy1024 = kHeld * 1024;
constexpr int kMostThreads = 1024;

// Threads of a row of `units` units, u a thread.
constexpr int threads_of(int64_t units, int u)
{
    const int64_t need = (units + u - 1) / u;
    return need <= 8 ? 8 : need <= 16 ? 16 : need <= 32 ? 32 : (int)((need + 63) / 64 * 64);
}

// T rows of `units` units each, at most `most` of them (a power of two) in a thread, where rows are read and written once: two units a thread, one for few rows. us, one / two / four units:
// bf16 norm with residual 16384 x 4096 88.3 / 90.1 / 92.9, 8192 x 1024 10.7 / 10.5 / -, 512 x 4096 4.1 / 4.0 / 4.4, 64 x 4096 3.1 / 3.1 / 3.7, 8192 x 4096 in 8 bits 41.9 / 41.6 / 46,
// 8192 x 11264 gated to 8 bits - / 86.7 / 105, 1 x 5632 2.8 / 3.2 / 3.8, float32 3001 x 1363 - / 10.6 / 10.9, 2048 x 768 - / 3.2 / 3.2.
// Rows of up to 32 units share a wave: 20000 x 64 bf16 8.3 us by a wave each, 4.4 so.
constexpr Plan plan_of(int64_t units, int most, int64_t T)
{
    int u = T > 64 && most > 1 && units > 32 ? 2 : 1;
    while (u < most && threads_of(units, u) > kMostThreads) u *= 2;
    const int threads = threads_of(units, u);
    return {u, threads, (T >= 1024 || threads < 64) && threads < 256 ? 256 / threads : 1};
}

// Where columns are summed over the rows as well (the norm's backward pass): one unit a thread as far as 16 waves have a row, work-groups of up to twelve waves and as many of them as the CUs hold at a
// time, each of which leaves a line of sums. us for work-groups so / of other numbers of waves and lines: 8192 x 4096 bf16 57.8 / 59 to 86, two units a thread 96; 8192 x 1024 - / 19.8 to 28,
// 3001 x 1363 float32 14.6 / 15 to 19.
struct BackwardPlan {
    Plan rows;
    int64_t lines;
};
constexpr BackwardPlan backward_plan_of(int64_t units, int most, int64_t T)
{
    int u = 1;
    while (u < most && threads_of(units, u) > kMostThreads) u *= 2;
    const int threads = threads_of(units, u), fit = threads < 768 ? 768 / threads : 1;
    const int rows = T >= 1024 ? fit : threads < 64 ? 64 / threads : 1;
    const int64_t groups = (T + rows - 1) / rows, held = 256 * (kMostThreads / (threads * rows));
    return {{u, threads, rows}, groups < held ? groups : held};
}

}  // namespace rows
}  // namespace anr
