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

// Rows in memory start at whole words, or (loose) anywhere, and end anywhere: they are loaded by whole words from the last one in front of them on, and what is read behind them (a next row, or zeros behind the
// last one, where the extent of the buffer's descriptor ends) is cleared in one of the operands, X.
//
// The first `count` bytes of an operand.
__device__ __forceinline__ void cut(i32x4& v, int count)
{
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const int bytes = min(max(count - 4 * j, 0), 4);
        v[j] &= bytes == 4 ? -1 : (int)((1u << (8 * bytes)) - 1u);
    }
}
// Sixteen bytes from byte `shift` % 4 on of `before` and v.
__device__ __forceinline__ i32x4 behind_byte(i32x4 v, int before, uint32_t shift)
{
    return i32x4{(int)__builtin_amdgcn_alignbyte(v[0], before, shift), (int)__builtin_amdgcn_alignbyte(v[1], v[0], shift), (int)__builtin_amdgcn_alignbyte(v[2], v[1], shift),
                 (int)__builtin_amdgcn_alignbyte(v[3], v[2], shift)};
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
// Four bytes a lane, alike.
__device__ __forceinline__ void load_word_to_lds(i32x4 descriptor, uint32_t offset, int step, uint32_t lds)
{
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dword %1, %2, %3 offen lds" ::"s"(lds), "v"(offset), "s"(descriptor), "s"(step) : "m0");
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
