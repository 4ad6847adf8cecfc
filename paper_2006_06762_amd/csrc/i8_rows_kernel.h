// Products of a few rows X [M,K], M <= 16 TB, of 8-bit integers with a large matrix W (i8_device.h), as single tokens need them.
//
// Bound: reading W once.  A work-group takes 16 rows of W, its waves share the k in chunks of 128 and join their sums in LDS; the matrix instructions
// (v_mfma_i32_16x16x64_i8) are sixteen tokens wide, which cost nothing here.
#pragma once
#include "gemm_i8_plan.h"
#include "i8_device.h"

namespace anr {
namespace i8 {

// The results of a thread: what they are multiplied with is read before the products, whose sums [wave][TB][4][64] join at the end.  At least four waves.
template <typename T, int TB>
struct Results {
    static constexpr int MOST = TB;
    float row[MOST], column[MOST], added[MOST];
    // register e of lane l: row 4 (l / 16) + e of W, token l % 16
    static __device__ __forceinline__ int token_of(int i) { return (i >> 8) * 16 + (i & 15); }
    static __device__ __forceinline__ int column_of(int i, int n0) { return n0 + 4 * ((i >> 4) & 3) + ((i >> 6) & 3); }
    __device__ __forceinline__ void init(const Args& a, int n0)
    {
#pragma unroll
        for (int j = 0; j < MOST; ++j) {
            const int i = threadIdx.x + j * (int)blockDim.x;
            row[j] = a.finish.of_row(min(token_of(i), a.M - 1));
            column[j] = a.finish.of_column(min(column_of(i, n0), a.N - 1));
            added[j] = a.finish.added(min(column_of(i, n0), a.N - 1));
        }
    }
    __device__ __forceinline__ void store(const Args& a, const int* sums, int n0) const
    {
        const int waves = blockDim.x >> 6;
#pragma unroll
        for (int j = 0; j < MOST; ++j) {
            const int i = threadIdx.x + j * (int)blockDim.x, token = token_of(i), n = column_of(i, n0);
            if (i >= TB * 256 || token >= a.M || n >= a.N) continue;
            int v = 0;
            for (int w = 0; w < waves; ++w) v += sums[w * TB * 256 + i];
            static_cast<T*>(a.d)[token * a.ldd + n] = from_float<T>(Finish::value(v, row[j], column[j], added[j]));
        }
    }
};

// Bytes of a wave's buffer: a chunk of its 16 rows of W and the 16 TB rows of X, and these rows' words in front of the chunk where they are loose.
template <int TB, bool LOOSE>
constexpr int stage_bytes() { return 16 * (1 + TB) * kRowsChunk + (LOOSE ? 512 : 0); }

// Rows go through LDS: a lane's operand is of one of sixteen rows, and loads whose neighbouring lanes are in different lines take four times as
// long to issue (32 tokens 4096 -> 11264 19.4 us straight from memory, so 13.6; 1 token 5632 -> 2048 5.4, 4.0).  Each wave has STAGES buffers of its own and waits for no other one but at the end.
// LOOSE: rows start at any byte, others at whole words.  They lie in LDS from their second word on, whose first starts up to three bytes ahead of them, and are put right when they are operands: sixteen
// bytes from the last word of the unit before on (through registers, by 16-byte loads at any address, which issue a lane a clock, 1 token 8193 -> 4096 10.4 us, so 8.1; 20 tokens 14.4, 10.4).
template <typename T, int TB, int STAGES, bool LOOSE>
__global__ __launch_bounds__(64 * most_waves(TB)) void stream_kernel(const Args a)
{
    constexpr int BK = kRowsChunk, STARTS = 16 * (1 + TB) * BK, STAGE = stage_bytes<TB, LOOSE>(), UNITS = 2 * (1 + TB), LOADS = UNITS + (LOOSE ? 2 : 0);
    extern __shared__ __attribute__((aligned(1024))) char lds[];                  // buffers, then sums [wave][TB][4][64]
    const uint32_t lds_at = settled(__builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)lds));
    const int tid = threadIdx.x, lane = tid & 63, wave = settled(__builtin_amdgcn_readfirstlane(tid >> 6)), waves = blockDim.x >> 6;
    const int n0 = blockIdx.x * 16, last_w = min(16, a.N - n0) - 1, last_x = a.M - 1;
    const int8_t* const w0 = a.w + n0 * a.ldw;
    // bytes of a word in front of the first rows
    const uint32_t ahead_w = LOOSE ? (uint32_t)reinterpret_cast<uintptr_t>(w0) & 3 : 0, ahead_x = LOOSE ? (uint32_t)reinterpret_cast<uintptr_t>(a.x) & 3 : 0;
    auto start_of = [&](bool x, int r) { return x ? ahead_x + (uint32_t)(min(r, last_x) * (int)a.ldx) : ahead_w + (uint32_t)(min(r, last_w) * (int)a.ldw); };
    // The extents end with the rows that exist: words past them are zeros.
    const i32x4 of_w = descriptor_of(w0 - ahead_w), of_x = descriptor_of(a.x - ahead_x);
    const int extent_w = settled(__builtin_amdgcn_readfirstlane((int)(ahead_w + last_w * (int)a.ldw + a.K + 3) & ~3));
    const int extent_x = settled(__builtin_amdgcn_readfirstlane((int)(ahead_x + last_x * (int)a.ldx + a.K + 3) & ~3));
    // A load is eight rows; a lane has one of these and one of its units
    uint32_t offset[UNITS], first_w = 0, first_x = 0;
#pragma unroll
    for (int i = 0; i < UNITS; ++i) {
        const int r = (i < 2 ? i : i - 2) * 8 + (lane >> 3);
        const uint32_t start = start_of(i >= 2, r);
        offset[i] = (LOOSE ? (start & ~3u) + 4 : start) + place_of<BK>(r, lane & 7) * kUnit;
    }
    if (LOOSE) {
        first_w = start_of(false, lane) & ~3u;
        first_x = start_of(true, lane) & ~3u;
    }
    const int chunks = (a.K + BK - 1) / BK;
    const uint32_t own = lds_at + wave * STAGES * STAGE;
    // (chunks past the last one read nothing)
    auto load = [&](int c, int stage) {
        i32x4 dw = of_w, dx = of_x;
        dw[2] = c < chunks ? extent_w : 0;
        dx[2] = c < chunks ? extent_x : 0;
        const uint32_t to = own + stage * STAGE;
#pragma unroll
        for (int i = 0; i < UNITS; ++i) load_to_lds(i < 2 ? dw : dx, offset[i], c * BK, to + i * 1024);
        if (LOOSE) {
            load_word_to_lds(dw, first_w, c * BK, to + STARTS);
            load_word_to_lds(dx, first_x, c * BK, to + STARTS + 256);
        }
    };
    uint32_t shift[1 + TB];
    if (LOOSE) {
#pragma unroll
        for (int j = 0; j < 1 + TB; ++j) shift[j] = start_of(j > 0, (j > 0 ? j - 1 : 0) * 16 + (lane & 15));
    }
    i32x4 acc[TB];
#pragma unroll
    for (int t = 0; t < TB; ++t) acc[t] = i32x4{0, 0, 0, 0};
    Results<T, TB> results;
    load(wave, 0);
    results.init(a, n0);                                             // (in front of the loads that the first wait leaves on their way)
#pragma unroll
    for (int s = 1; s < STAGES; ++s) load(wave + s * waves, s);
    int stage = 0;
#pragma unroll 1
    for (int c = wave; c < chunks; c += waves) {
        wait_for_loads<(STAGES - 1) * LOADS>();
        const char* const at = lds + (wave * STAGES + stage) * STAGE;
        i32x4 v[2][1 + TB];
        int before[2][1 + TB];
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int j = 0; j < 1 + TB; ++j) {
                const int r = lane & 15, u = 4 * i + (lane >> 4);
                const char* const row = at + (j * 16 + r) * BK;
                v[i][j] = *reinterpret_cast<const i32x4*>(row + place_of<BK>(r, u) * kUnit);
                if (LOOSE) before[i][j] = *reinterpret_cast<const int*>(u > 0 ? row + place_of<BK>(r, u - 1) * kUnit + 12 : at + STARTS + (j > 0 ? 256 + (j - 1) * 64 : 0) + r * 4);
            }
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        load(c + STAGES * waves, stage);
        stage = stage + 1 == STAGES ? 0 : stage + 1;
        if (LOOSE) {
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int j = 0; j < 1 + TB; ++j) v[i][j] = behind_byte(v[i][j], before[i][j], shift[j]);
        }
        if ((c + 1) * BK > a.K) {
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int t = 0; t < TB; ++t) cut(v[i][1 + t], a.K - c * BK - (4 * i + (lane >> 4)) * kUnit);
        }
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int t = 0; t < TB; ++t) acc[t] = __builtin_amdgcn_mfma_i32_16x16x64_i8(v[i][0], v[i][1 + t], acc[t], 0, 0, 0);
    }
    wait_for_loads<0>();
    __syncthreads();
    int* const sums = reinterpret_cast<int*>(lds);
#pragma unroll
    for (int t = 0; t < TB; ++t)
#pragma unroll
        for (int e = 0; e < 4; ++e) sums[((wave * TB + t) * 4 + e) * 64 + lane] = acc[t][e];
    __syncthreads();
    results.store(a, sums, n0);
}

}  // namespace i8
}  // namespace anr
