// What the kernels of products of 8-bit integers share: D[m][n] = (sum_k X[m][k] W[n][k]) x_scale[m] w_scale[n] + bias[n], both operands rows of k.
// The sums are exact (32 bits hold k < 2^17 products of magnitudes up to 128); a result takes the rounding of the sum to 24 bits, two of the scales, one of
// the bias and that to its type.
#pragma once
#include "anr_kernels.h"
#include "element_types.h"

namespace anr {
namespace i8 {

typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef int i32x16 __attribute__((ext_vector_type(16)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

constexpr int kUnit = 16;                       // k of a lane's operand
constexpr uint32_t kNowhere = 0x80000000u;      // byte offset past every descriptor's extent: loads zeros
constexpr int kExtent = 0x7fffffff;

// Scales and bias, each of which may be absent.
struct Finish {
    const float *x_scale, *w_scale;
    const void* bias;
    int bias_dtype;
    __device__ __forceinline__ float of_row(int64_t m) const { return x_scale ? x_scale[m] : 1.f; }
    __device__ __forceinline__ float of_column(int64_t n) const { return w_scale ? w_scale[n] : 1.f; }
    __device__ __forceinline__ float added(int64_t n) const { return bias ? load_any(bias, n, bias_dtype) : 0.f; }
    // (a sum with zero leaves everything but the sign of zero as it is)
    static __device__ __forceinline__ float value(int sum, float row, float column, float added) { return (float)sum * row * column + added; }
};

struct Args {
    const int8_t *x, *w;
    void* d;
    int64_t ldx, ldw, ldd;
    int M, N, K;
    Finish finish;
    int tiles_m, tiles_n;
    int band;                       // tiles are walked in bands of so many rows of tiles
    int splits;                     // work-groups that share a tile's k: their sums go to `parts`, [split][M][N] packed
    int* parts;
    bool streaming;                 // D's stores go past L2: a wave's part of a row is whole lines of 128 bytes
};

// Sixteen values of k of a row, from k on; those past K are cleared by `clear` where they were read.  Not WHOLE (pointers, leading dimensions and K are any): the
// row's last unit starts so far ahead that it ends with the row (K >= 16), and the values that it shares with the unit before are cleared in one of the operands,
// X: other values of k in their place, in both operands alike.
__device__ __forceinline__ int loose_start(int k, int K) { return min(k, K - kUnit); }
__device__ __forceinline__ u32x4 load_loose(const int8_t* p)
{
    struct __attribute__((packed, aligned(1))) Loose { u32x4 v; };
    return reinterpret_cast<const Loose*>(p)->v;
}
__device__ __forceinline__ void clear_counted(u32x4& v, int k, int K)
{
    const int counted = min(k - loose_start(k, K), kUnit);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int bytes = min(max(counted - 4 * i, 0), 4);
        v[i] &= bytes == 4 ? 0u : 0xffffffffu << (8 * bytes);
    }
}

// The unit of a row in LDS that holds the row's unit u.
template <int BK>
__device__ __forceinline__ int place_of(int row, int u) { return BK == 128 ? u ^ ((row >> 1) & 7) : u ^ ((row >> 2) & 3); }

// Sixteen bytes a lane from memory to LDS, in the order of the lanes from `lds` on: lane l's from byte offset + step of the descriptor's extent.  The lanes'
// registers are read when the instruction is issued and none is written; s_waitcnt vmcnt and a barrier come before LDS is read.  In asm, because the
// compiler has every LDS read that follows such a load wait for all of them.
__device__ __forceinline__ void load_to_lds(i32x4 descriptor, uint32_t offset, int step, uint32_t lds)
{
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, %3 offen lds" ::"s"(lds), "v"(offset), "s"(descriptor), "s"(step) : "m0");
}
// A scalar register that the vector unit wrote is read by a memory instruction five cycles later at the earliest, which the compiler sees to for its own instructions only: what
// load_to_lds takes comes from here, and what is made of it stays in the scalar unit.
template <typename V>
__device__ __forceinline__ V settled(V v)
{
    asm volatile("s_nop 4" : "+s"(v));
    return v;
}
template <int OUTSTANDING>
__device__ __forceinline__ void wait_for_loads()
{
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(OUTSTANDING) : "memory");
}
__device__ __forceinline__ i32x4 descriptor_of(const void* p)
{
    const uint64_t at = reinterpret_cast<uint64_t>(p);
    return settled(i32x4{__builtin_amdgcn_readfirstlane((int)at), __builtin_amdgcn_readfirstlane((int)(at >> 32) & 0xffff), kExtent, 0x00020000});
}

}  // namespace i8
}  // namespace anr
