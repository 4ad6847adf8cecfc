// Launch interface between the C-ABI layer and the operators of a transformer block (group norm, rotary positions, gated
// feed-forward).  As in anr_kernels.h: arguments are validated, launchers neither allocate nor synchronise.
#pragma once
#include "anr.h"
#include "anr_kernels.h"

namespace anr {

struct GroupNormArgs {
    const void* x;
    const void* dy;                 // backward only
    void* y;                        // forward: y, backward: dx (may be null)
    const void *gamma, *beta;       // null: ones, zeros
    void *dgamma, *dbeta;           // backward only (may be null)
    float *mean, *rstd;             // outputs of the forward (may be null), inputs of the backward call
    float eps;
    int N, H, W, C, groups, act, dtype, param_dtype;
    int64_t xs[3], dys[3], ys[3];   // strides (n, h, w); ys: those of `y` above
    void* ws;
};
size_t group_norm_workspace_bytes(const GroupNormArgs& a, bool backward);
hipError_t launch_group_norm(const GroupNormArgs& a, hipStream_t stream);
hipError_t launch_group_norm_backward(const GroupNormArgs& a, hipStream_t stream);

struct RotaryArgs {
    const void *q, *k;
    void *q_out, *k_out;
    const void* positions;
    const float* inv_freq;
    anr_rotary_desc d;              // strides filled in
};
hipError_t launch_rotary(const RotaryArgs& a, hipStream_t stream);

struct GatedFfArgs {
    const void *x, *dy, *w_gate, *w_up, *w_down;
    void* y;
    void *gate, *up;                // outputs of the forward (may be null), inputs of the backward call
    void *dx, *dw_gate, *dw_up, *dw_down;
    anr_gated_ff_desc d;            // leading dimensions filled in
    void* ws;
};
size_t gated_ff_workspace_bytes(const GatedFfArgs& a, bool backward);
hipError_t launch_gated_ff(const GatedFfArgs& a, hipStream_t stream);
hipError_t launch_gated_ff_backward(const GatedFfArgs& a, hipStream_t stream);

// The status of a launch, noted for anr_last_hip_error (api.cpp).
anr_status launch_result(hipError_t e);
// anr_workspace_size for the operators above (api_blocks.cpp).
anr_status blocks_workspace_size(int op, const void* desc, size_t* bytes);

}  // namespace anr
