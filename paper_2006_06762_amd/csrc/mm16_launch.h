// Launches of mm16_kernel.h for one element type (mm16_f16.hip, mm16_bf16.hip).
#pragma once
#include "mm16_kernel.h"

namespace anr {
namespace mm16 {

// The products of the gated feed-forward block: kinds of the operands and what becomes of the sums.
enum Form {
    FORM_GATED,          // x (rows of k) by gate's and up's weights (rows of k)
    FORM_ROWS,           // both operands rows of k, stored
    FORM_HIDDEN_GRADS,   // dy (rows of k) by w_down (columns of k): dg, du, h
    FORM_INPUT_GRAD,     // dg, du (rows of k) by gate's and up's weights (columns of k)
    FORM_WEIGHT_GRADS    // both operands columns of k
};

// A work-group's tile, and whether two groups of waves share its k.
enum Shape { SHAPE_256, SHAPE_128, SHAPE_128_TWICE };
constexpr int edge_of(Shape s) { return s == SHAPE_256 ? 256 : 128; }

hipError_t launch_products_f16(Form form, Shape shape, bool aligned, const Args& a, hipStream_t stream);
hipError_t launch_products_bf16(Form form, Shape shape, bool aligned, const Args& a, hipStream_t stream);

template <typename T, int BM, int BN, int WM, int WN, int G, Kind XK, Kind WK, Epilogue EPI, bool ALIGNED>
hipError_t launch_one(const Args& a, hipStream_t stream)
{
    static LdsLimit limit;
    auto* const kernel = product_kernel<T, BM, BN, WM, WN, G, XK, WK, EPI, ALIGNED>;
    constexpr size_t lds = G * lds_bytes<BM, BN, XK, WK>();
    const hipError_t e = raise_lds_limit(reinterpret_cast<const void*>(kernel), lds, limit);
    if (e != hipSuccess) return e;
    return launch_kernel(kernel, dim3((unsigned)(a.first_tile[a.problems] * a.splits)), dim3(64 * WM * WN * G), lds, stream, a);
}

// 256 x 256: with both operands rows of k four waves of 128 x 128 (gate and up of 8192 x 4096 -> 11264 in 1.17 ms, eight waves of 128 x 64,
// which read half as much again from LDS, 1.46), else eight (operands turned in LDS: level, and the backward epilogue has no registers
// beside 128 x 128 sums).
template <typename T, Kind XK, Kind WK, Epilogue EPI, bool ALIGNED>
hipError_t launch_shape(Shape shape, const Args& a, hipStream_t stream)
{
    constexpr int WIDE = XK == K_ROWS && WK == K_ROWS ? 2 : 4;
    if (shape == SHAPE_256) return launch_one<T, 256, 256, 2, WIDE, 1, XK, WK, EPI, ALIGNED>(a, stream);
    if (shape == SHAPE_128_TWICE) return launch_one<T, 128, 128, 2, 2, 2, XK, WK, EPI, ALIGNED>(a, stream);
    return launch_one<T, 128, 128, 2, 2, 1, XK, WK, EPI, ALIGNED>(a, stream);
}
template <typename T, Kind XK, Kind WK, Epilogue EPI>
hipError_t launch_tile(Shape shape, bool aligned, const Args& a, hipStream_t stream)
{
    return aligned ? launch_shape<T, XK, WK, EPI, true>(shape, a, stream) : launch_shape<T, XK, WK, EPI, false>(shape, a, stream);
}

template <typename T>
hipError_t launch_products(Form form, Shape shape, bool aligned, const Args& a, hipStream_t stream)
{
    switch (form) {
        case FORM_GATED: return launch_tile<T, K_ROWS, K_ROWS, GATED>(shape, aligned, a, stream);
        case FORM_HIDDEN_GRADS: return launch_tile<T, K_ROWS, K_COLUMNS, GATED_BACKWARD>(shape, aligned, a, stream);
        case FORM_INPUT_GRAD: return a.splits > 1 ? launch_tile<T, K_ROWS, K_COLUMNS, PARTIAL>(shape, aligned, a, stream)
                                                  : launch_tile<T, K_ROWS, K_COLUMNS, STORE>(shape, aligned, a, stream);
        case FORM_WEIGHT_GRADS: return launch_tile<T, K_COLUMNS, K_COLUMNS, STORE>(shape, aligned, a, stream);
        default: return a.splits > 1 ? launch_tile<T, K_ROWS, K_ROWS, PARTIAL>(shape, aligned, a, stream)
                                     : launch_tile<T, K_ROWS, K_ROWS, STORE>(shape, aligned, a, stream);
    }
}

}  // namespace mm16
}  // namespace anr
