// C-ABI layer of the operators of a transformer block: argument validation (host only, before any launch) and dispatch.
// See include/anr.h for the contract of every entry point.
#include <algorithm>
#include <cmath>

#include "anr.h"
#include "blocks_internal.h"
#include "element_types.h"

namespace {

// A stride of 2^40 elements, or one that takes its extent beyond 2^58: below both no offset, nor the sum of three, overflows.
bool far(int64_t stride, int64_t extent) { return stride >= (int64_t)1 << 40 || stride >= ((int64_t)1 << 58) / extent; }

bool valid_type(int t) { return t == ANR_F32 || t == ANR_F16 || t == ANR_BF16; }
bool valid_act(int a) { return a >= ANR_ACT_NONE && a <= ANR_ACT_GELU_TANH; }
bool element_aligned(const void* p, int dtype) { return (reinterpret_cast<uintptr_t>(p) & (uintptr_t)(anr::element_bytes(dtype) - 1)) == 0; }
bool all_zero(const int64_t s[3]) { return s[0] == 0 && s[1] == 0 && s[2] == 0; }

// Whether no two elements of a view meet: `inner` neighbouring ones, three extents with their strides in any order.
bool apart(const int64_t (&extent)[3], const int64_t (&stride)[3], int64_t inner)
{
    if (extent[0] == 0 || extent[1] == 0 || extent[2] == 0) return true;
    int order[3] = {0, 1, 2};
    std::sort(order, order + 3, [&](int a, int b) { return stride[a] < stride[b]; });
    int64_t span = inner;
    for (int i : order) {
        if (extent[i] <= 1) continue;
        if (stride[i] < span) return false;
        span += (extent[i] - 1) * stride[i];
    }
    return true;
}

// A call's workspace.
anr_status check_workspace(const void* ws, size_t ws_bytes, size_t need)
{
    if (need == 0) return ANR_OK;
    if (!ws || ws_bytes < need) return ANR_ERR_WORKSPACE;
    return anr::is_aligned16(ws) ? ANR_OK : ANR_ERR_INVALID_ARG;
}

// ---- group norm

anr_status check_group_norm(const anr_group_norm_desc* d, bool backward, anr::GroupNormArgs* a)
{
    if (!d) return ANR_ERR_NULL;
    if (d->N < 0 || d->H < 0 || d->W < 0 || d->C < 1 || d->groups < 1 || d->C % d->groups != 0) return ANR_ERR_INVALID_ARG;
    if (!valid_act(d->act) || !valid_type(d->dtype) || (d->param_dtype != ANR_F32 && d->param_dtype != d->dtype)) return ANR_ERR_INVALID_ARG;
    // chunks of channels and images are extents of the grid; pixels are counted in 32 bits, a step beyond the last one too
    if (d->N >= 65535 || d->C > 1 << 20 || d->C / d->groups > 8192 || (int64_t)d->H * d->W > (int64_t)1 << 30) return ANR_ERR_UNSUPPORTED;
    const int64_t extent[3] = {d->N, d->H, d->W};
    const int64_t* const in[3] = {d->x_stride, d->y_stride, d->dx_stride};
    int64_t* const out[3] = {a->xs, backward ? a->dys : a->ys, a->ys};
    for (int t = 0; t < (backward ? 3 : 2); ++t) {
        int64_t s[3] = {in[t][0], in[t][1], in[t][2]};
        if (all_zero(s)) {
            s[2] = d->C;
            s[1] = d->W * s[2];
            s[0] = d->H * s[1];
        } else {
            for (int i = 0; i < 3; ++i) {
                if (extent[i] <= 1) continue;
                if (s[i] < 1) return ANR_ERR_INVALID_ARG;
                if (far(s[i], extent[i])) return ANR_ERR_UNSUPPORTED;
            }
            if (!apart(extent, s, d->C)) return ANR_ERR_INVALID_ARG;
        }
        // the strides of single extents say nothing: those of a packed neighbour, so that they stand in no kernel's way
        if (d->W <= 1) s[2] = d->H > 1 ? s[1] : d->C;
        if (d->H <= 1) s[1] = d->W * s[2];
        if (d->N <= 1) s[0] = 0;
        for (int i = 0; i < 3; ++i) out[t][i] = s[i];
    }
    a->N = d->N;
    a->H = d->H;
    a->W = d->W;
    a->C = d->C;
    a->groups = d->groups;
    a->act = d->act;
    a->dtype = d->dtype;
    a->param_dtype = d->param_dtype;
    return ANR_OK;
}

bool same_strides(const int64_t* a, const int64_t* b) { return a[0] == b[0] && a[1] == b[1] && a[2] == b[2]; }

bool empty(const anr::GroupNormArgs& a) { return a.N == 0 || a.H == 0 || a.W == 0; }

// ---- rotary positions

anr_status check_rotary(const anr_rotary_desc* d, anr_rotary_desc* out)
{
    if (!d) return ANR_ERR_NULL;
    if (d->B < 0 || d->S < 0 || d->H < 0 || d->Hk < 0 || d->D < 1 || d->axes < 1 || d->axes > 4) return ANR_ERR_INVALID_ARG;
    int64_t pairs = 0;
    for (int i = 0; i < d->axes; ++i) {
        if (d->section[i] < 0) return ANR_ERR_INVALID_ARG;
        pairs += d->section[i];
    }
    if (2 * pairs > d->D || !valid_type(d->dtype) || d->pairing < ANR_ROTARY_HALVES || d->pairing > ANR_ROTARY_SECTION_HALVES) return ANR_ERR_INVALID_ARG;
    if (d->inverse < 0 || d->inverse > 1 || d->pos_type < ANR_POS_I32 || d->pos_type > ANR_POS_F32 || d->reserved != 0) return ANR_ERR_INVALID_ARG;
    // a grid has 2^32 threads, of which a token can take 256
    if (d->D > 2048 || (int64_t)d->H + d->Hk > 65536 || (int64_t)d->B * d->S >= (int64_t)1 << 24) return ANR_ERR_UNSUPPORTED;
    *out = *d;
    int64_t* const strides[4] = {out->q_stride, out->k_stride, out->q_out_stride, out->k_out_stride};
    for (int t = 0; t < 4; ++t) {
        const int64_t heads = t & 1 ? d->Hk : d->H;
        int64_t* const s = strides[t];
        if (all_zero(s)) {
            s[2] = d->D;
            s[1] = heads * s[2];
            s[0] = d->S * s[1];
        }
        const int64_t extent[3] = {d->B, d->S, heads}, given[3] = {s[0], s[1], s[2]};
        for (int i = 0; i < 3; ++i) {
            if (extent[i] <= 1) {
                s[i] = 0;
                continue;
            }
            if (s[i] < 0) return ANR_ERR_INVALID_ARG;
            if (far(s[i], extent[i])) return ANR_ERR_UNSUPPORTED;
        }
        if (t >= 2 && !apart(extent, given, d->D)) return ANR_ERR_INVALID_ARG;
    }
    const int64_t extent[3] = {d->axes, d->B, d->S};
    for (int i = 0; i < 3; ++i) {
        if (extent[i] <= 1) {
            out->pos_stride[i] = 0;
            continue;
        }
        if (out->pos_stride[i] < 0) return ANR_ERR_INVALID_ARG;
        if (far(out->pos_stride[i], extent[i])) return ANR_ERR_UNSUPPORTED;
    }
    return ANR_OK;
}

// ---- gated feed-forward block

anr_status check_gated_ff(const anr_gated_ff_desc* d, anr_gated_ff_desc* out)
{
    if (!d) return ANR_ERR_NULL;
    if (d->T < 0 || d->C < 1 || d->F < 1 || !valid_act(d->act) || !valid_type(d->dtype)) return ANR_ERR_INVALID_ARG;
    // the kernels' 32-bit offsets inside a tile, and the grids of the float32 products
    if (d->C > 1 << 20 || d->F > 1 << 20 || d->T >= 1 << 22) return ANR_ERR_UNSUPPORTED;
    *out = *d;
    int64_t* const ld[8] = {&out->ldx, &out->ldy, &out->ldpre, &out->lddx, &out->ldw, &out->ld_down, &out->lddw, &out->ld_ddown};
    const int64_t least[8] = {d->C, d->C, d->F, d->C, d->C, d->F, d->C, d->F};
    for (int i = 0; i < 8; ++i) {
        if (*ld[i] == 0) *ld[i] = least[i];
        if (*ld[i] < least[i]) return ANR_ERR_INVALID_ARG;
        if (*ld[i] >= 1 << 22) return ANR_ERR_UNSUPPORTED;
    }
    return ANR_OK;
}

// ---- root-mean-square norm

// Leading dimensions of matrices of T rows: 0 is packed; those of a single row say nothing.
anr_status fill_leading(int64_t T, int n, int64_t* const* ld, const int64_t* least)
{
    for (int i = 0; i < n; ++i) {
        if (*ld[i] == 0) *ld[i] = least[i];
        if (T <= 1 && *ld[i] >= 0) *ld[i] = least[i];
        if (*ld[i] < least[i]) return ANR_ERR_INVALID_ARG;
        if (far(*ld[i], T > 0 ? T : 1)) return ANR_ERR_UNSUPPORTED;
    }
    return ANR_OK;
}

anr_status check_rms_norm(const anr_rms_norm_desc* d, anr_rms_norm_desc* out)
{
    if (!d) return ANR_ERR_NULL;
    if (d->T < 0 || d->C < 1 || !valid_type(d->dtype) || (d->param_dtype != ANR_F32 && d->param_dtype != d->dtype)) return ANR_ERR_INVALID_ARG;
    // a row is held in the registers of one work-group
    if (d->C > 32768 || d->T >= (int64_t)1 << 31) return ANR_ERR_UNSUPPORTED;
    *out = *d;
    int64_t* const ld[4] = {&out->ldx, &out->ld_residual, &out->ldh, &out->ldy};
    const int64_t least[4] = {d->C, d->C, d->C, d->C};
    return fill_leading(d->T, 4, ld, least);
}

// Whether an output is one of the inputs with another leading dimension.
struct Matrix {
    const void* p;
    int64_t ld;
};
bool crossed(Matrix out, std::initializer_list<Matrix> inputs)
{
    for (const Matrix& in : inputs)
        if (out.p && out.p == in.p && out.ld != in.ld) return true;
    return false;
}

// What the two forward calls have in common.
anr_status rms_norm_forward_args(const anr_rms_norm_desc* d, const void* x, const void* residual, const void* gamma, float eps, void* h, void* y, anr::RmsNormArgs* a)
{
    const anr_status st = check_rms_norm(d, &a->d);
    if (st != ANR_OK) return st;
    if (!std::isfinite(eps) || eps < 0.f || (h && !residual)) return ANR_ERR_INVALID_ARG;
    if (d->T > 0 && (!x || !y)) return ANR_ERR_NULL;
    if (!element_aligned(x, d->dtype) || !element_aligned(residual, d->dtype) || !element_aligned(h, d->dtype) || !element_aligned(gamma, d->param_dtype)) return ANR_ERR_INVALID_ARG;
    if (crossed({h, a->d.ldh}, {{x, a->d.ldx}, {residual, a->d.ld_residual}}) || (h && h == y)) return ANR_ERR_INVALID_ARG;
    a->x = x;
    a->residual = residual;
    a->gamma = gamma;
    a->eps = eps;
    a->h = h;
    a->y = y;
    return ANR_OK;
}

// ---- rows in 8 bits

anr_status check_rows_q8(const anr_rows_q8_desc* d, bool back, anr_rows_q8_desc* out)
{
    if (!d) return ANR_ERR_NULL;
    if (d->T < 0 || d->C < 1 || !valid_type(d->dtype) || !valid_act(d->act) || (back && d->act != ANR_ACT_NONE)) return ANR_ERR_INVALID_ARG;
    if (d->C > 1 << 20 || d->T >= (int64_t)1 << 31) return ANR_ERR_UNSUPPORTED;
    *out = *d;
    int64_t* const ld[3] = {&out->ldx, &out->ldq, &out->ld_up};
    const int64_t least[3] = {d->C, d->C, d->C};
    return fill_leading(d->T, back ? 2 : 3, ld, least);
}

// ---- products of 8-bit integers

anr_status check_gemm_i8(const anr_gemm_i8_desc* d, anr_gemm_i8_desc* out)
{
    if (!d) return ANR_ERR_NULL;
    if (d->M < 0 || d->N < 1 || d->K < 1 || !valid_type(d->dtype) || (d->bias_dtype != ANR_F32 && d->bias_dtype != d->dtype)) return ANR_ERR_INVALID_ARG;
    // sums in 32 bits, and the kernels' 32-bit offsets inside a tile
    if (d->K >= 1 << 17 || d->N > 1 << 20 || d->M >= 1 << 22) return ANR_ERR_UNSUPPORTED;
    *out = *d;
    const int64_t rows[3] = {d->M, d->N, d->M}, least[3] = {d->K, d->K, d->N};
    int64_t* const ld[3] = {&out->lda, &out->ldw, &out->ldd};
    for (int i = 0; i < 3; ++i) {
        const anr_status st = fill_leading(rows[i], 1, &ld[i], &least[i]);
        if (st != ANR_OK) return st;
        if (*ld[i] >= 1 << 22) return ANR_ERR_UNSUPPORTED;
    }
    return ANR_OK;
}

}  // namespace

namespace anr {

anr_status blocks_workspace_size(int op, const void* desc, size_t* bytes)
{
    GroupNormArgs gn{};
    RotaryArgs r{};
    GatedFfArgs ff{};
    RmsNormArgs rn{};
    RowsQ8Args rq{};
    GemmI8Args gi{};
    anr_status st = ANR_ERR_INVALID_ARG;
    switch (op) {
        case ANR_OP_GROUP_NORM:
        case ANR_OP_GROUP_NORM_BACKWARD:
            st = check_group_norm(static_cast<const anr_group_norm_desc*>(desc), op == ANR_OP_GROUP_NORM_BACKWARD, &gn);
            if (st == ANR_OK) *bytes = group_norm_workspace_bytes(gn, op == ANR_OP_GROUP_NORM_BACKWARD);
            break;
        case ANR_OP_ROTARY:
            st = check_rotary(static_cast<const anr_rotary_desc*>(desc), &r.d);
            if (st == ANR_OK) *bytes = 0;
            break;
        case ANR_OP_GATED_FF:
        case ANR_OP_GATED_FF_BACKWARD:
            st = check_gated_ff(static_cast<const anr_gated_ff_desc*>(desc), &ff.d);
            if (st == ANR_OK) *bytes = gated_ff_workspace_bytes(ff, op == ANR_OP_GATED_FF_BACKWARD);
            break;
        case ANR_OP_RMS_NORM:
        case ANR_OP_RMS_NORM_Q8:
        case ANR_OP_RMS_NORM_BACKWARD:
            st = check_rms_norm(static_cast<const anr_rms_norm_desc*>(desc), &rn.d);
            if (st == ANR_OK) *bytes = op == ANR_OP_RMS_NORM_BACKWARD ? rms_norm_backward_workspace_bytes(rn) : 0;
            break;
        case ANR_OP_QUANTIZE_ROWS:
        case ANR_OP_DEQUANTIZE_ROWS:
            st = check_rows_q8(static_cast<const anr_rows_q8_desc*>(desc), op == ANR_OP_DEQUANTIZE_ROWS, &rq.d);
            if (st == ANR_OK) *bytes = 0;
            break;
        case ANR_OP_GEMM_I8:
            st = check_gemm_i8(static_cast<const anr_gemm_i8_desc*>(desc), &gi.d);
            if (st == ANR_OK) *bytes = gemm_i8_workspace_bytes(gi);
            break;
        default: break;
    }
    return st;
}

}  // namespace anr

extern "C" {

anr_status anr_group_norm(const anr_group_norm_desc* d, const void* x, const void* gamma, const void* beta, float eps, void* y, float* mean, float* rstd, void* ws,
                          size_t ws_bytes, void* hip_stream)
{
    anr::GroupNormArgs a{};
    anr_status st = check_group_norm(d, false, &a);
    if (st != ANR_OK) return st;
    if (!std::isfinite(eps) || eps < 0.f) return ANR_ERR_INVALID_ARG;
    if (!empty(a) && (!x || !y)) return ANR_ERR_NULL;
    if (!element_aligned(x, d->dtype) || !element_aligned(y, d->dtype) || !element_aligned(gamma, d->param_dtype) || !element_aligned(beta, d->param_dtype) ||
        !element_aligned(mean, ANR_F32) || !element_aligned(rstd, ANR_F32))
        return ANR_ERR_INVALID_ARG;
    if (x && x == y && !same_strides(a.xs, a.ys)) return ANR_ERR_INVALID_ARG;
    st = check_workspace(ws, ws_bytes, anr::group_norm_workspace_bytes(a, false));
    if (st != ANR_OK) return st;
    a.x = x;
    a.y = y;
    a.gamma = gamma;
    a.beta = beta;
    a.mean = mean;
    a.rstd = rstd;
    a.eps = eps;
    a.ws = ws;
    return anr::launch_result(anr::launch_group_norm(a, static_cast<hipStream_t>(hip_stream)));
}

anr_status anr_group_norm_backward(const anr_group_norm_desc* d, const void* dy, const void* x, const void* gamma, const void* beta, const float* mean, const float* rstd,
                                   void* dx, void* dgamma, void* dbeta, void* ws, size_t ws_bytes, void* hip_stream)
{
    anr::GroupNormArgs a{};
    anr_status st = check_group_norm(d, true, &a);
    if (st != ANR_OK) return st;
    if (!dx && !dgamma && !dbeta && !empty(a)) return ANR_ERR_NULL;
    if (!empty(a) && (!dy || !x || !mean || !rstd)) return ANR_ERR_NULL;
    if (!element_aligned(dy, d->dtype) || !element_aligned(x, d->dtype) || !element_aligned(dx, d->dtype) || !element_aligned(gamma, d->param_dtype) ||
        !element_aligned(beta, d->param_dtype) || !element_aligned(dgamma, d->param_dtype) || !element_aligned(dbeta, d->param_dtype) || !element_aligned(mean, ANR_F32) ||
        !element_aligned(rstd, ANR_F32))
        return ANR_ERR_INVALID_ARG;
    if (dx && ((dx == x && !same_strides(a.xs, a.ys)) || (dx == dy && !same_strides(a.dys, a.ys)))) return ANR_ERR_INVALID_ARG;
    st = check_workspace(ws, ws_bytes, anr::group_norm_workspace_bytes(a, true));
    if (st != ANR_OK) return st;
    a.dy = dy;
    a.x = x;
    a.y = dx;
    a.gamma = gamma;
    a.beta = beta;
    a.dgamma = dgamma;
    a.dbeta = dbeta;
    a.mean = const_cast<float*>(mean);
    a.rstd = const_cast<float*>(rstd);
    a.ws = ws;
    return anr::launch_result(anr::launch_group_norm_backward(a, static_cast<hipStream_t>(hip_stream)));
}

anr_status anr_rotary(const anr_rotary_desc* d, const void* q, const void* k, const void* positions, const float* inv_freq, void* q_out, void* k_out, void* ws,
                      size_t ws_bytes, void* hip_stream)
{
    (void)ws; (void)ws_bytes;
    anr::RotaryArgs a{};
    const anr_status st = check_rotary(d, &a.d);
    if (st != ANR_OK) return st;
    const bool tokens = d->B > 0 && d->S > 0;
    int pairs = 0;
    for (int i = 0; i < d->axes; ++i) pairs += d->section[i];
    if (tokens && ((d->H > 0 && (!q || !q_out)) || (d->Hk > 0 && (!k || !k_out)))) return ANR_ERR_NULL;
    if (tokens && pairs > 0 && d->H + d->Hk > 0 && (!positions || !inv_freq)) return ANR_ERR_NULL;
    if (!element_aligned(q, d->dtype) || !element_aligned(k, d->dtype) || !element_aligned(q_out, d->dtype) || !element_aligned(k_out, d->dtype) ||
        !element_aligned(inv_freq, ANR_F32) || (reinterpret_cast<uintptr_t>(positions) & (d->pos_type == ANR_POS_I64 ? 7 : 3)) != 0)
        return ANR_ERR_INVALID_ARG;
    if ((q && q == q_out && !same_strides(a.d.q_stride, a.d.q_out_stride)) || (k && k == k_out && !same_strides(a.d.k_stride, a.d.k_out_stride))) return ANR_ERR_INVALID_ARG;
    a.q = q;
    a.k = k;
    a.positions = positions;
    a.inv_freq = inv_freq;
    a.q_out = q_out;
    a.k_out = k_out;
    return anr::launch_result(anr::launch_rotary(a, static_cast<hipStream_t>(hip_stream)));
}

anr_status anr_gated_ff(const anr_gated_ff_desc* d, const void* x, const void* w_gate, const void* w_up, const void* w_down, void* y, void* gate, void* up, void* ws,
                        size_t ws_bytes, void* hip_stream)
{
    anr::GatedFfArgs a{};
    anr_status st = check_gated_ff(d, &a.d);
    if (st != ANR_OK) return st;
    if (d->T > 0 && (!x || !w_gate || !w_up || !w_down || !y || (!gate != !up))) return ANR_ERR_NULL;
    for (const void* p : {x, w_gate, w_up, w_down, static_cast<const void*>(y), static_cast<const void*>(gate), static_cast<const void*>(up)})
        if (!element_aligned(p, d->dtype)) return ANR_ERR_INVALID_ARG;
    st = check_workspace(ws, ws_bytes, anr::gated_ff_workspace_bytes(a, false));
    if (st != ANR_OK) return st;
    a.x = x;
    a.w_gate = w_gate;
    a.w_up = w_up;
    a.w_down = w_down;
    a.y = y;
    a.gate = gate;
    a.up = up;
    a.ws = ws;
    return anr::launch_result(anr::launch_gated_ff(a, static_cast<hipStream_t>(hip_stream)));
}

anr_status anr_gated_ff_backward(const anr_gated_ff_desc* d, const void* dy, const void* x, const void* w_gate, const void* w_up, const void* w_down, const void* gate,
                                 const void* up, void* dx, void* dw_gate, void* dw_up, void* dw_down, void* ws, size_t ws_bytes, void* hip_stream)
{
    anr::GatedFfArgs a{};
    anr_status st = check_gated_ff(d, &a.d);
    if (st != ANR_OK) return st;
    if (d->T > 0 && (!dy || !x || !w_gate || !w_up || !w_down || !gate || !up)) return ANR_ERR_NULL;
    if (d->T > 0 && !dx && !dw_gate && !dw_up && !dw_down) return ANR_ERR_NULL;
    for (const void* p : {dy, x, w_gate, w_up, w_down, gate, up, static_cast<const void*>(dx), static_cast<const void*>(dw_gate), static_cast<const void*>(dw_up),
                          static_cast<const void*>(dw_down)})
        if (!element_aligned(p, d->dtype)) return ANR_ERR_INVALID_ARG;
    st = check_workspace(ws, ws_bytes, anr::gated_ff_workspace_bytes(a, true));
    if (st != ANR_OK) return st;
    a.dy = dy;
    a.x = x;
    a.w_gate = w_gate;
    a.w_up = w_up;
    a.w_down = w_down;
    a.gate = const_cast<void*>(gate);
    a.up = const_cast<void*>(up);
    a.dx = dx;
    a.dw_gate = dw_gate;
    a.dw_up = dw_up;
    a.dw_down = dw_down;
    a.ws = ws;
    return anr::launch_result(anr::launch_gated_ff_backward(a, static_cast<hipStream_t>(hip_stream)));
}

anr_status anr_rms_norm(const anr_rms_norm_desc* d, const void* x, const void* residual, const void* gamma, float eps, void* h, void* y, float* rstd, void* ws,
                        size_t ws_bytes, void* hip_stream)
{
    (void)ws; (void)ws_bytes;
    anr::RmsNormArgs a{};
    const anr_status st = rms_norm_forward_args(d, x, residual, gamma, eps, h, y, &a);
    if (st != ANR_OK) return st;
    if (!element_aligned(y, d->dtype) || !element_aligned(rstd, ANR_F32)) return ANR_ERR_INVALID_ARG;
    if (crossed({y, a.d.ldy}, {{x, a.d.ldx}, {residual, a.d.ld_residual}})) return ANR_ERR_INVALID_ARG;
    a.rstd = rstd;
    return anr::launch_result(anr::launch_rms_norm(a, static_cast<hipStream_t>(hip_stream)));
}

anr_status anr_rms_norm_q8(const anr_rms_norm_desc* d, const void* x, const void* residual, const void* gamma, float eps, void* h, int8_t* q, float* scale, void* ws,
                           size_t ws_bytes, void* hip_stream)
{
    (void)ws; (void)ws_bytes;
    anr::RmsNormArgs a{};
    const anr_status st = rms_norm_forward_args(d, x, residual, gamma, eps, h, q, &a);
    if (st != ANR_OK) return st;
    if (d->T > 0 && !scale) return ANR_ERR_NULL;
    if (!element_aligned(scale, ANR_F32) || (q && (q == x || q == residual))) return ANR_ERR_INVALID_ARG;
    a.scale = scale;
    return anr::launch_result(anr::launch_rms_norm_q8(a, static_cast<hipStream_t>(hip_stream)));
}

anr_status anr_rms_norm_backward(const anr_rms_norm_desc* d, const void* dy, const void* x, const void* gamma, const float* rstd, const void* dh, void* dx, void* dgamma,
                                 void* ws, size_t ws_bytes, void* hip_stream)
{
    anr::RmsNormArgs a{};
    anr_status st = check_rms_norm(d, &a.d);
    if (st != ANR_OK) return st;
    if (d->T > 0 && (!dy || !x || !rstd || (!dx && !dgamma))) return ANR_ERR_NULL;
    for (const void* p : {dy, x, dh, static_cast<const void*>(dx)})
        if (!element_aligned(p, d->dtype)) return ANR_ERR_INVALID_ARG;
    if (!element_aligned(gamma, d->param_dtype) || !element_aligned(dgamma, d->param_dtype) || !element_aligned(rstd, ANR_F32)) return ANR_ERR_INVALID_ARG;
    if (crossed({dx, a.d.ldh}, {{dy, a.d.ldy}, {x, a.d.ldx}, {dh, a.d.ld_residual}})) return ANR_ERR_INVALID_ARG;
    st = check_workspace(ws, ws_bytes, anr::rms_norm_backward_workspace_bytes(a));
    if (st != ANR_OK) return st;
    a.dy = dy;
    a.x = x;
    a.gamma = gamma;
    a.rstd = const_cast<float*>(rstd);
    a.residual = dh;
    a.h = dx;
    a.dgamma = dgamma;
    a.ws = ws;
    return anr::launch_result(anr::launch_rms_norm_backward(a, static_cast<hipStream_t>(hip_stream)));
}

anr_status anr_quantize_rows(const anr_rows_q8_desc* d, const void* x, const void* up, int8_t* q, float* scale, void* ws, size_t ws_bytes, void* hip_stream)
{
    (void)ws; (void)ws_bytes;
    anr::RowsQ8Args a{};
    const anr_status st = check_rows_q8(d, false, &a.d);
    if (st != ANR_OK) return st;
    if (d->T > 0 && (!x || !q || !scale)) return ANR_ERR_NULL;
    if (!element_aligned(x, d->dtype) || !element_aligned(up, d->dtype) || !element_aligned(scale, ANR_F32) || (q && (q == x || q == up))) return ANR_ERR_INVALID_ARG;
    a.x = x;
    a.up = up;
    a.q = q;
    a.scale = scale;
    return anr::launch_result(anr::launch_quantize_rows(a, static_cast<hipStream_t>(hip_stream)));
}

anr_status anr_dequantize_rows(const anr_rows_q8_desc* d, const int8_t* q, const float* scale, void* y, void* ws, size_t ws_bytes, void* hip_stream)
{
    (void)ws; (void)ws_bytes;
    anr::RowsQ8Args a{};
    const anr_status st = check_rows_q8(d, true, &a.d);
    if (st != ANR_OK) return st;
    if (d->T > 0 && (!q || !scale || !y)) return ANR_ERR_NULL;
    if (!element_aligned(y, d->dtype) || !element_aligned(scale, ANR_F32) || (y && y == q)) return ANR_ERR_INVALID_ARG;
    a.x = y;
    a.q = const_cast<int8_t*>(q);
    a.scale = const_cast<float*>(scale);
    return anr::launch_result(anr::launch_dequantize_rows(a, static_cast<hipStream_t>(hip_stream)));
}

anr_status anr_gemm_i8(const anr_gemm_i8_desc* d, const int8_t* a, const int8_t* w, const float* a_scale, const float* w_scale, const void* bias, void* out, void* ws,
                       size_t ws_bytes, void* hip_stream)
{
    anr::GemmI8Args g{};
    anr_status st = check_gemm_i8(d, &g.d);
    if (st != ANR_OK) return st;
    if (d->M > 0 && (!a || !w || !out)) return ANR_ERR_NULL;
    if (!element_aligned(out, d->dtype) || !element_aligned(a_scale, ANR_F32) || !element_aligned(w_scale, ANR_F32) || !element_aligned(bias, d->bias_dtype) ||
        (out && (out == a || out == w || out == a_scale || out == w_scale || out == bias)))
        return ANR_ERR_INVALID_ARG;
    st = check_workspace(ws, ws_bytes, anr::gemm_i8_workspace_bytes(g));
    if (st != ANR_OK) return st;
    g.a = a;
    g.w = w;
    g.a_scale = a_scale;
    g.w_scale = w_scale;
    g.bias = bias;
    g.out = out;
    g.ws = ws;
    return anr::launch_result(anr::launch_gemm_i8(g, static_cast<hipStream_t>(hip_stream)));
}

}  // extern "C"
