// Values joined over the lanes of a wave.
#pragma once
#include <hip/hip_runtime.h>

namespace anr {

// A lane's value from another one of its row of 16, or (ROWS: a mask of the rows that take it, zero in the others) the last one of a row before.
template <int CONTROL, int ROWS, typename T>
__device__ __forceinline__ T of_lane(T v)
{
    constexpr int WORDS = sizeof(T) / 4;
    struct Words { int w[WORDS]; } from = __builtin_bit_cast(Words, v), to;
#pragma unroll
    for (int i = 0; i < WORDS; ++i) to.w[i] = __builtin_amdgcn_update_dpp(0, from.w[i], CONTROL, ROWS, 0xf, false);
    return __builtin_bit_cast(T, to);
}

// All lanes' values joined by `join`, for which zero is neutral, by lanes that read each other's registers; always in the same order.
template <typename T, typename Join>
__device__ __forceinline__ T wave_join(T v, Join join)
{
    v = join(v, of_lane<0xb1, 0xf>(v));         // pairs: quad_perm 1, 0, 3, 2
    v = join(v, of_lane<0x4e, 0xf>(v));         // fours: quad_perm 2, 3, 0, 1
    v = join(v, of_lane<0x141, 0xf>(v));        // eights: row_half_mirror
    v = join(v, of_lane<0x140, 0xf>(v));        // sixteens: row_mirror
    v = join(v, of_lane<0x142, 0xa>(v));        // row_bcast 15: rows 1 and 3 hold two rows
    v = join(v, of_lane<0x143, 0xc>(v));        // row_bcast 31: row 3 holds all
    constexpr int WORDS = sizeof(T) / 4;
    struct Words { int w[WORDS]; } all = __builtin_bit_cast(Words, v);
#pragma unroll
    for (int i = 0; i < WORDS; ++i) all.w[i] = __builtin_amdgcn_readlane(all.w[i], 63);
    return __builtin_bit_cast(T, all);
}

// The same over each run of 8, 16 or 32 lanes.
template <typename T, typename Join>
__device__ __forceinline__ T lanes_join(T v, int lanes, Join join)
{
    v = join(v, of_lane<0xb1, 0xf>(v));
    v = join(v, of_lane<0x4e, 0xf>(v));
    v = join(v, of_lane<0x141, 0xf>(v));
    if (lanes > 8) v = join(v, of_lane<0x140, 0xf>(v));
    if (lanes > 16) v = join(v, __shfl_xor(v, 16));
    return v;
}

template <typename T>
__device__ __forceinline__ T wave_sum(T v)
{
    return wave_join(v, [](T a, T b) { return a + b; });
}
__device__ __forceinline__ uint32_t wave_max(uint32_t v)
{
    return wave_join(v, [](uint32_t a, uint32_t b) { return a > b ? a : b; });
}

}  // namespace anr
