// Rows of C values that the threads of one or more waves hold in registers, for operators that go over a row more than once but read it
// once: sums or largest values of the row, then every value of it again.
//
// Unit i of a row are its V values (16 bytes) from i V on; a thread has units t, t + threads, and so on, so that a wave reads 1 KB at a time.
// The last unit of a row whose length is no whole number of units starts so far ahead that it ends with the row: its first values are another
// unit's too, which both compute and store alike, and which only the sums have to leave out.  No load stands under a branch.  Values that
// start at any element's address are read and written 16 bytes at a time as well, which the memory pipes take.
// Rows of less than one unit have units of one value.
#pragma once
#include "element_types.h"
#include "wave_join.h"

namespace anr {
namespace rows {

constexpr int kMostWaves = 16;                   // of a work-group

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4_loose __attribute__((ext_vector_type(4), aligned(2)));     // at any element's address

// V values as they lie in memory, at any element's address.
template <typename T, int V>
struct Raw {
    static constexpr int BYTES = sizeof(T) * V;
    static constexpr int WORDS = BYTES >= 4 ? BYTES / 4 : 1;
    uint32_t w[WORDS];

    __device__ __forceinline__ void load(const T* p)
    {
        if constexpr (V == 1) {
            w[0] = 0;
            __builtin_memcpy(w, p, sizeof(T));
        } else {
            struct __attribute__((packed, aligned(sizeof(T)))) Loose { uint32_t w[WORDS]; };
            const Loose l = *reinterpret_cast<const Loose*>(p);
#pragma unroll
            for (int i = 0; i < WORDS; ++i) w[i] = l.w[i];
        }
    }
    __device__ __forceinline__ void fill(T v)
    {
        T a[V];
#pragma unroll
        for (int i = 0; i < V; ++i) a[i] = v;
        w[0] = 0;
        __builtin_memcpy(w, a, sizeof a);
    }
    // What is converted before and after this is converted twice: between, only the values as they lie in memory take registers.
    __device__ __forceinline__ void keep_packed()
    {
#pragma unroll
        for (int i = 0; i < WORDS; ++i) asm("" : "+v"(w[i]));
    }
    __device__ __forceinline__ void floats(float (&out)[V]) const
    {
        T a[V];
        __builtin_memcpy(a, w, sizeof a);
#pragma unroll
        for (int i = 0; i < V; ++i) out[i] = to_float(a[i]);
    }
};

// STREAMING: past L2 (see stg4_nt), at any element's address as well (4096 x 4003 bf16 with its residual 30 us by ordinary stores, 21 so; 16384 x 1001 25.1, 21.5).
template <bool STREAMING, typename T, int V>
__device__ __forceinline__ void store(T* p, const float (&v)[V])
{
    const Pack<T, V> a = pack_floats<T, V>(v);
    if constexpr (STREAMING && sizeof(T) * V >= 16) {
#pragma unroll
        for (int i = 0; i < (int)sizeof(T) * V / 16; ++i) {
            u32x4 w;
            __builtin_memcpy(&w, reinterpret_cast<const char*>(&a) + 16 * i, 16);
            __builtin_nontemporal_store(w, reinterpret_cast<u32x4_loose*>(p) + i);
        }
    } else {
        struct __attribute__((packed, aligned(sizeof(T)))) Loose { T v[V]; };
        Loose l;
#pragma unroll
        for (int i = 0; i < V; ++i) l.v[i] = a.v[i];
        *reinterpret_cast<Loose*>(p) = l;
    }
}

// Where unit i of a row of C values starts, and how many of its values another unit counts (V: all of them, it is past the end).
template <int V, bool WHOLE>
struct Unit {
    int start, counted;
    __device__ __forceinline__ Unit(int i, int C)
    {
        const int64_t own = (int64_t)i * V;
        start = (int)(own < C - V ? own : C - V);
        counted = WHOLE ? (own < C ? 0 : V) : (int)(own - start < V ? own - start : V);
    }
    __device__ __forceinline__ bool in() const { return counted < V; }
    __device__ __forceinline__ bool counts(int j) const { return WHOLE ? counted == 0 : j >= counted; }
};

// Element i of a row: an offset of 32 bits from the row's address, which is a scalar where whole waves have a row.
template <typename T>
__device__ __forceinline__ const T* at(const void* row, int i)
{
    return reinterpret_cast<const T*>(static_cast<const char*>(row) + (uint32_t)i * (uint32_t)sizeof(T));
}
template <typename T>
__device__ __forceinline__ T* at(void* row, int i)
{
    return reinterpret_cast<T*>(static_cast<char*>(row) + (uint32_t)i * (uint32_t)sizeof(T));
}

// A row's number (below 2^31), in a scalar register where whole waves have it, so that its addresses are not in as many vector registers.
template <bool WAVES>
__device__ __forceinline__ int64_t row_of(int64_t row) { return WAVES ? (int64_t)__builtin_amdgcn_readfirstlane((int)row) : row; }

// The bits of |v|, whose order as whole numbers is that of the magnitudes, infinity and NaN above all others.
__device__ __forceinline__ uint32_t magnitude(float v) { return __builtin_bit_cast(uint32_t, v) & 0x7fffffffu; }
constexpr uint32_t kInfinite = 0x7f800000u;

// A row in 8 bits: whole steps of `step`, the largest magnitude of the row being 127 of them.  Rows of zeros have the step zero, whatever the factor; an infinity or NaN
// makes the step NaN, so that whatever is made of the row is NaN.  Values are zeros where the step is none that they could be divided by: zero (a 127th of what is below 2^-143 rounds to it) or NaN.  Rows that lie low in float32's range are raised before they are
// divided by their step, whose inverse would leave it at the other end.
struct Steps {
    float inverse, rest;            // their sum is the inverse of the step of the (raised) values, to 2^-45 of itself; to 2^-29 at the upper end of the range, where `rest` is denormal
    bool raised;
    float step;                     // of rows whose values are multiplied by `factor` afterwards
    __device__ __forceinline__ Steps(uint32_t largest, float factor)
    {
        const float most = __builtin_bit_cast(float, largest), result = largest == 0 ? 0.f : most * factor;
        const bool fine = magnitude(result) < kInfinite;
        raised = most < 0x1p-60f;
        const float unit = (raised ? most * 0x1p64f : most) / 127.f;
        inverse = fine && result >= 0x1p-143f ? __builtin_amdgcn_rcpf(unit) : 0.f;
        rest = fmaf(-inverse, unit, 1.f) * inverse;
        step = fine ? result / 127.f : __builtin_nanf("");
    }
};

// V of them at any address.  The quotient by the step is off by less than 2^-28 of itself before it is rounded to 24 bits, and so exact where they hold it: half a step stays
// one (by `inverse` alone one of two halves came out on its wrong side, as 1.5 in steps of 3; 8192 x 11264 bf16 gated 84.3 us, so 85.7, 8192 x 4096 normed with its residual 42.1, 42.1, 1024 x 32768 62.2, 64.7).  It is rounded to a
// whole number, ties to even, by a sum with 1.5 2^23, whose last bits are then that number's (at most 127 + 2^-16).
template <int V>
__device__ __forceinline__ void store_steps(int8_t* p, float (&v)[V], const Steps& steps)
{
    if (steps.raised) {
#pragma unroll
        for (int i = 0; i < V; ++i) v[i] *= 0x1p64f;
    }
    auto bits = [&](int i) { return __builtin_bit_cast(uint32_t, fmaf(v[i], steps.inverse, v[i] * steps.rest) + 12582912.f); };
    if constexpr (V == 1) {
        p[0] = steps.inverse == 0.f ? (int8_t)0 : (int8_t)bits(0);
    } else {
        struct __attribute__((packed, aligned(1))) Loose { uint32_t w[V / 4]; };
        Loose l;
#pragma unroll
        for (int i = 0; i < V / 4; ++i) {
            const uint32_t low = __builtin_amdgcn_perm(bits(4 * i + 1), bits(4 * i), 0x0c0c0400u), high = __builtin_amdgcn_perm(bits(4 * i + 3), bits(4 * i + 2), 0x04000c0cu);
            l.w[i] = steps.inverse == 0.f ? 0u : low | high;
        }
        *reinterpret_cast<Loose*>(p) = l;
    }
}

// A sum and a largest magnitude over the threads of a row (blockDim.x: whole waves, or 8, 16 or 32 lanes of one; a work-group has blockDim.y rows), those of both that are
// asked for. `round` alternates from call to call, so that one barrier is enough.
struct Joined {
    float sum;
    uint32_t largest;
};
template <bool SUM, bool LARGEST>
__device__ __forceinline__ Joined join_row(Joined v, int round)
{
    __shared__ Joined parts[2][kMostWaves];
    if (blockDim.x < 64) {
        if (SUM) v.sum = lanes_join(v.sum, blockDim.x, [](float a, float b) { return a + b; });
        if (LARGEST) v.largest = lanes_join(v.largest, blockDim.x, [](uint32_t a, uint32_t b) { return a > b ? a : b; });
        return v;
    }
    if (SUM) v.sum = wave_sum(v.sum);
    if (LARGEST) v.largest = wave_max(v.largest);
    const int waves = blockDim.x >> 6;
    if (waves == 1) return v;
    const int first = threadIdx.y * waves, wave = threadIdx.x >> 6;
    if ((threadIdx.x & 63) == 0) parts[round][first + wave] = v;
    __syncthreads();
    v = parts[round][first];
    for (int i = 1; i < waves; ++i) {
        if (SUM) v.sum += parts[round][first + i].sum;
        if (LARGEST) v.largest = max(v.largest, parts[round][first + i].largest);
    }
    return v;
}

}  // namespace rows
}  // namespace anr
