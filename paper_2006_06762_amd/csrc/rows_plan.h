// How rows of C values are dealt to waves (rows_device.h): plain arithmetic without a device in it.
#pragma once
#include <stdint.h>

namespace anr {
namespace rows {

struct Plan {
    int units;                      // of a thread: a power of two
    int waves;                      // of a row
    int rows;                       // of a work-group
};

constexpr int kHeld = 32;           // floats of a thread in work-groups of up to 1024 threads
constexpr int kHeldBy1024 = kHeld * 1024;

// Rows of `units` units of V values each, T of them; at most `most` units a thread.
constexpr Plan plan_of(int64_t units, int most, int64_t T)
{
    const int wanted = T >= 1024 ? 4 : 16;       // waves that a row may have
    int u = 1;
    while (u < most && (units + 64 * u - 1) / (64 * u) > wanted) u *= 2;
    const int waves = (int)((units + 64 * u - 1) / (64 * u));
    return {u, waves, T >= 1024 && waves < 4 ? 4 / waves : 1};
}

}  // namespace rows
}  // namespace anr
