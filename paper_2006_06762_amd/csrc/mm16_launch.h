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

hipError_t launch_products_f16(Form form, int tile, bool aligned, const Args& a, hipStream_t stream);
hipError_t launch_products_bf16(Form form, int tile, bool aligned, const Args& a, hipStream_t stream);

template <typename T, int BM, int BN, int WM, int WN, Kind XK, Kind WK, Epilogue EPI, bool ALIGNED>
hipError_t launch_one(const Args& a, hipStream_t stream)
{
    static LdsLimit limit;
    auto* const kernel = product_kernel<T, BM, BN, WM, WN, XK, WK, EPI, ALIGNED>;
    constexpr size_t lds = lds_bytes<BM, BN, XK, WK>();
    const hipError_t e = raise_lds_limit(reinterpret_cast<const void*>(kernel), lds, limit);
    if (e != hipSuccess) return e;
    return launch_kernel(kernel, dim3((unsigned)(a.first_tile[a.problems] * a.splits)), dim3(64 * WM * WN), lds, stream, a);
}

template <typename T, Kind XK, Kind WK, Epilogue EPI>
hipError_t launch_tile(int tile, bool aligned, const Args& a, hipStream_t stream)
{
    if (tile == 256)
        return aligned ? launch_one<T, 256, 256, 2, 4, XK, WK, EPI, true>(a, stream) : launch_one<T, 256, 256, 2, 4, XK, WK, EPI, false>(a, stream);
    return aligned ? launch_one<T, 128, 128, 2, 2, XK, WK, EPI, true>(a, stream) : launch_one<T, 128, 128, 2, 2, XK, WK, EPI, false>(a, stream);
}

template <typename T>
hipError_t launch_products(Form form, int tile, bool aligned, const Args& a, hipStream_t stream)
{
    switch (form) {
        case FORM_GATED: return launch_tile<T, K_ROWS, K_ROWS, GATED>(tile, aligned, a, stream);
        case FORM_HIDDEN_GRADS: return launch_tile<T, K_ROWS, K_COLUMNS, GATED_BACKWARD>(tile, aligned, a, stream);
        case FORM_INPUT_GRAD: return a.splits > 1 ? launch_tile<T, K_ROWS, K_COLUMNS, PARTIAL>(tile, aligned, a, stream)
                                                  : launch_tile<T, K_ROWS, K_COLUMNS, STORE>(tile, aligned, a, stream);
        case FORM_WEIGHT_GRADS: return launch_tile<T, K_COLUMNS, K_COLUMNS, STORE>(tile, aligned, a, stream);
        default: return a.splits > 1 ? launch_tile<T, K_ROWS, K_ROWS, PARTIAL>(tile, aligned, a, stream)
                                     : launch_tile<T, K_ROWS, K_ROWS, STORE>(tile, aligned, a, stream);
    }
}

}  // namespace mm16
}  // namespace anr
