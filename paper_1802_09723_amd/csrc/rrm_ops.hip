// C entries of the operators between and behind the linear layers: checks of the arguments, then the launches.
#include "op_common.h"

using namespace rrm;

namespace {

// Elements [i][j][0 .. c) of an output, at i * outer + j * inner: no two at one place, none below the pointer.
bool apart(int64_t rows_outer, int64_t outer, int64_t rows_inner, int64_t inner, int64_t c) {
    if (rows_outer < 1 || rows_inner < 1 || c < 1) return true;
    if ((rows_outer > 1 && outer < c) || (rows_inner > 1 && inner < c)) return false;
    if (rows_outer == 1 || rows_inner == 1) return true;
    // one axis lies within a step of the other (strides below 2^40, rows below 2^31: nothing overflows when divided)
    return outer - c >= 0 && inner - c >= 0 && ((outer - c) / inner >= rows_inner - 1 || (inner - c) / outer >= rows_outer - 1);
}
// strides that keep every offset within 62 bits
bool reachable(int64_t rows_outer, int64_t outer, int64_t rows_inner, int64_t inner) {
    const int64_t lim = (int64_t)1 << 60;
    const int64_t o = outer < 0 ? -(outer + 1) : outer, i = inner < 0 ? -(inner + 1) : inner;  // (no overflow at the type's lowest)
    return o <= lim / (rows_outer > 0 ? rows_outer : 1) && i <= lim / (rows_inner > 0 ? rows_inner : 1);
}
bool misaligned(const void* p, size_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) != 0; }
size_t elem_bytes(int elem) { return elem == RRM_F32 ? 4 : 2; }

rrm_status finish(hipError_t e) {
    return e == hipSuccess ? RRM_OK : record_failure(RRM_ERR_HIP, hipGetErrorString(e));
}

rrm_status check_workspace(const void* ws, size_t have, size_t need) {
    if (need == 0) return RRM_OK;
    if (!ws) return record_failure(RRM_ERR_NULL, "workspace is NULL");
    if (misaligned(ws, 256)) return record_failure(RRM_ERR_ALIGN, "workspace is not 256-byte aligned");
    if (have < need) return record_failure(RRM_ERR_WORKSPACE, "workspace is smaller than the *_workspace function says");
    return RRM_OK;
}

rrm_status check_act(int act) {
    if (act < RRM_ACT_NONE || act > RRM_ACT_GELU) return record_failure(RRM_ERR_OPTION, "unknown activation");
    return RRM_OK;
}

rrm_status check(const rrm_norm_desc* d) {
    if (!d) return record_failure(RRM_ERR_NULL, "desc is NULL");
    if (d->x_elem < RRM_F32 || d->x_elem > RRM_BF16 || d->y_elem < RRM_F32 || d->y_elem > RRM_BF16)
        return record_failure(RRM_ERR_DTYPE, "group norm: elements are RRM_F32 or RRM_BF16");
    if (d->n < 0 || d->positions < 0 || d->c < 1 || d->groups < 1 || d->c % d->groups)
        return record_failure(RRM_ERR_SHAPE, "group norm: n and positions not negative, c positive, groups a divisor of c");
    // (below 2^31 by more than any kernel's step over channels or positions)
    if ((int64_t)d->n * d->c > 0x7ffff000 || d->positions > 0x7ffff000)
        return record_failure(RRM_ERR_SHAPE, "group norm: n * c and positions are at most 2^31 - 4096");
    if (!(d->eps > 0.0f) || d->eps > 3.0e38f) return record_failure(RRM_ERR_OPTION, "group norm: eps must be positive and finite");
    return check_act(d->act);
}

rrm_status check(const rrm_scan_desc* d) {
    if (!d) return record_failure(RRM_ERR_NULL, "desc is NULL");
    if (d->elem < RRM_F32 || d->elem > RRM_BF16) return record_failure(RRM_ERR_DTYPE, "gated scan: elements are RRM_F32 or RRM_BF16");
    if (d->n < 0 || d->t < 0 || d->c < 0) return record_failure(RRM_ERR_SHAPE, "gated scan: n, t, c must not be negative");
    if (d->t > 0x7fffff00) return record_failure(RRM_ERR_SHAPE, "gated scan: t is at most 2^31 - 256");
    if ((int64_t)d->n * d->c > 0x7fffffff) return record_failure(RRM_ERR_SHAPE, "gated scan: n * c must fit 31 bits");
    return RRM_OK;
}

rrm_status check(const rrm_ff_desc* d) {
    if (!d) return record_failure(RRM_ERR_NULL, "desc is NULL");
    if (d->m < 0 || d->k < 1 || d->f < 1) return record_failure(RRM_ERR_SHAPE, "feed-forward: m not negative, k and f positive");
    if (d->m > (1 << 27) || d->k > (1 << 24) || d->f > (1 << 24)) return record_failure(RRM_ERR_SHAPE, "feed-forward: m up to 2^27, k and f up to 2^24");
    if ((int64_t)d->m * d->k > (1ll << 40) || (int64_t)d->m * d->f > (1ll << 40) || (int64_t)d->f * d->k > (1ll << 40))
        return record_failure(RRM_ERR_SHAPE, "feed-forward: tensors of up to 2^40 elements");
    return check_act(d->act);
}

}  // namespace

extern "C" {
#pragma GCC visibility push(default)

size_t rrm_group_norm_workspace(const rrm_norm_desc* desc, int backward) {
    if (check(desc) != RRM_OK || desc->n == 0 || desc->positions == 0) return 0;
    return norm_scratch(*desc, backward != 0);
}

rrm_status rrm_group_norm_act(const rrm_norm_desc* desc, const void* x, const float* gamma, const float* beta, void* y,
                              float* stats, void* workspace, size_t workspace_bytes, void* hip_stream) {
    if (rrm_status st = check(desc)) return st;
    const rrm_norm_desc& d = *desc;
    if (d.n == 0 || d.positions == 0) return RRM_OK;
    if (!x || !y) return record_failure(RRM_ERR_NULL, "x / y is NULL");
    if (!reachable(d.n, d.x_sample, d.positions, d.x_position) || !reachable(d.n, d.y_sample, d.positions, d.y_position))
        return record_failure(RRM_ERR_SHAPE, "group norm: strides out of range");
    if (!apart(d.n, d.y_sample, d.positions, d.y_position, d.c))
        return record_failure(RRM_ERR_SHAPE, "group norm: two elements of y lie at one place");
    if (misaligned(x, elem_bytes(d.x_elem)) || misaligned(y, elem_bytes(d.y_elem)) || misaligned(gamma, 4) || misaligned(beta, 4) ||
        misaligned(stats, 4))
        return record_failure(RRM_ERR_ALIGN, "group norm: a pointer is not aligned to its element");
    if (rrm_status st = check_workspace(workspace, workspace_bytes, norm_scratch(d, false))) return st;
    return finish(launch_group_norm(d, x, gamma, beta, y, stats, workspace, static_cast<hipStream_t>(hip_stream)));
}

rrm_status rrm_group_norm_act_backward(const rrm_norm_desc* desc, const void* x, const float* stats, const float* gamma,
                                       const float* beta, const void* dy, void* dx, float* dgamma, float* dbeta,
                                       void* workspace, size_t workspace_bytes, void* hip_stream) {
    if (rrm_status st = check(desc)) return st;
    const rrm_norm_desc& d = *desc;
    const bool some = d.n > 0 && d.positions > 0;
    if (some && (!x || !dy || !stats)) return record_failure(RRM_ERR_NULL, "x / dy / stats is NULL");
    if (!dgamma && !dbeta && (!dx || !some)) return RRM_OK;
    if (!reachable(d.n, d.x_sample, d.positions, d.x_position) || !reachable(d.n, d.y_sample, d.positions, d.y_position) ||
        !reachable(d.n, d.dx_sample, d.positions, d.dx_position))
        return record_failure(RRM_ERR_SHAPE, "group norm: strides out of range");
    if (dx && !apart(d.n, d.dx_sample, d.positions, d.dx_position, d.c))
        return record_failure(RRM_ERR_SHAPE, "group norm: two elements of dx lie at one place");
    if (misaligned(x, elem_bytes(d.x_elem)) || misaligned(dy, elem_bytes(d.y_elem)) || misaligned(dx, elem_bytes(d.x_elem)) ||
        misaligned(gamma, 4) || misaligned(beta, 4) || misaligned(stats, 4) || misaligned(dgamma, 4) || misaligned(dbeta, 4))
        return record_failure(RRM_ERR_ALIGN, "group norm: a pointer is not aligned to its element");
    if (some)
        if (rrm_status st = check_workspace(workspace, workspace_bytes, norm_scratch(d, true))) return st;
    return finish(launch_group_norm_backward(d, x, stats, gamma, beta, dy, dx, dgamma, dbeta, workspace,
                                             static_cast<hipStream_t>(hip_stream)));
}

int rrm_scan_marks(int t) { return t < 1 ? 0 : (t - 1) / RRM_SCAN_MARK_FRAMES + 1; }

size_t rrm_gated_scan_workspace(const rrm_scan_desc* desc, int backward) {
    if (check(desc) != RRM_OK || desc->n == 0 || desc->c == 0 || desc->t == 0) return 0;
    return scan_scratch(*desc, backward != 0);
}

rrm_status rrm_gated_scan(const rrm_scan_desc* desc, const void* x, const void* f, const float* h0, const int32_t* lengths,
                          void* y, float* h_last, float* marks, void* workspace, size_t workspace_bytes, void* hip_stream) {
    if (rrm_status st = check(desc)) return st;
    const rrm_scan_desc& d = *desc;
    if (d.n == 0 || d.c == 0) return RRM_OK;
    if (d.t > 0 && (!x || !f || !y)) return record_failure(RRM_ERR_NULL, "x / f / y is NULL");
    if (!reachable(d.n, d.x_video, d.t, d.x_frame) || !reachable(d.n, d.f_video, d.t, d.f_frame) ||
        !reachable(d.n, d.y_video, d.t, d.y_frame))
        return record_failure(RRM_ERR_SHAPE, "gated scan: strides out of range");
    if (!apart(d.n, d.y_video, d.t, d.y_frame, d.c)) return record_failure(RRM_ERR_SHAPE, "gated scan: two elements of y lie at one place");
    if (h_last && h_last == h0 && d.t > 1) return record_failure(RRM_ERR_STATE, "gated scan: h_last may be h0 for one frame only");
    const size_t e = elem_bytes(d.elem);
    if (misaligned(x, e) || misaligned(f, e) || misaligned(y, e) || misaligned(h0, 4) || misaligned(lengths, 4) ||
        misaligned(h_last, 4) || misaligned(marks, 4))
        return record_failure(RRM_ERR_ALIGN, "gated scan: a pointer is not aligned to its element");
    if (d.t > 0)
        if (rrm_status st = check_workspace(workspace, workspace_bytes, scan_scratch(d, false))) return st;
    return finish(launch_gated_scan(d, x, f, h0, lengths, y, h_last, marks, workspace, static_cast<hipStream_t>(hip_stream)));
}

rrm_status rrm_gated_scan_backward(const rrm_scan_desc* desc, const void* x, const void* f, const float* marks,
                                   const int32_t* lengths, const void* dy, const float* dh_last, void* dx, void* df,
                                   float* dh0, void* workspace, size_t workspace_bytes, void* hip_stream) {
    if (rrm_status st = check(desc)) return st;
    const rrm_scan_desc& d = *desc;
    if (d.n == 0 || d.c == 0) return RRM_OK;
    if (d.t > 0 && (!x || !f || !marks || !dy || !dx || !df)) return record_failure(RRM_ERR_NULL, "x / f / marks / dy / dx / df is NULL");
    if (!reachable(d.n, d.x_video, d.t, d.x_frame) || !reachable(d.n, d.f_video, d.t, d.f_frame) ||
        !reachable(d.n, d.y_video, d.t, d.y_frame) || !reachable(d.n, d.dx_video, d.t, d.dx_frame) ||
        !reachable(d.n, d.df_video, d.t, d.df_frame))
        return record_failure(RRM_ERR_SHAPE, "gated scan: strides out of range");
    if (!apart(d.n, d.dx_video, d.t, d.dx_frame, d.c) || !apart(d.n, d.df_video, d.t, d.df_frame, d.c))
        return record_failure(RRM_ERR_SHAPE, "gated scan: two elements of dx or of df lie at one place");
    const size_t e = elem_bytes(d.elem);
    if (misaligned(x, e) || misaligned(f, e) || misaligned(dy, e) || misaligned(dx, e) || misaligned(df, e) || misaligned(marks, 4) ||
        misaligned(lengths, 4) || misaligned(dh_last, 4) || misaligned(dh0, 4))
        return record_failure(RRM_ERR_ALIGN, "gated scan: a pointer is not aligned to its element");
    if (d.t > 0)
        if (rrm_status st = check_workspace(workspace, workspace_bytes, scan_scratch(d, true))) return st;
    return finish(launch_gated_scan_backward(d, x, f, marks, lengths, dy, dh_last, dx, df, dh0, workspace,
                                             static_cast<hipStream_t>(hip_stream)));
}

size_t rrm_gated_ff_workspace(const rrm_ff_desc* desc, int backward) {
    if (check(desc) != RRM_OK) return 0;
    return ff_scratch(*desc, backward != 0);
}

rrm_status rrm_gated_ff(const rrm_ff_desc* desc, const void* x, const void* wg, const void* wu, void* h, void* g, void* u,
                        void* workspace, size_t workspace_bytes, void* hip_stream) {
    if (rrm_status st = check(desc)) return st;
    const rrm_ff_desc& d = *desc;
    if (d.m == 0) return RRM_OK;
    if (!x || !wg || !wu || !h) return record_failure(RRM_ERR_NULL, "x / wg / wu / h is NULL");
    if ((g == nullptr) != (u == nullptr)) return record_failure(RRM_ERR_NULL, "g and u are kept together");
    if (!reachable(1, 0, d.m, d.x_row) || !reachable(1, 0, d.f, d.wg_row) || !reachable(1, 0, d.f, d.wu_row) ||
        !reachable(1, 0, d.m, d.h_row) || !reachable(1, 0, d.m, d.gu_row))
        return record_failure(RRM_ERR_SHAPE, "feed-forward: strides out of range");
    if (!apart(1, 0, d.m, d.h_row, d.f) || (g && !apart(1, 0, d.m, d.gu_row, d.f)))
        return record_failure(RRM_ERR_SHAPE, "feed-forward: two elements of an output lie at one place");
    const size_t e = d.unaligned ? 2 : 16;
    if (misaligned(x, e) || misaligned(wg, e) || misaligned(wu, e) || misaligned(h, 2) || misaligned(g, 2) || misaligned(u, 2))
        return record_failure(RRM_ERR_ALIGN, "feed-forward: a pointer is not aligned (to 16 bytes, to its element: see rrm_ff_desc)");
    if (rrm_status st = check_workspace(workspace, workspace_bytes, ff_scratch(d, false))) return st;
    return finish(launch_gated_ff(d, x, wg, wu, h, g, u, workspace, static_cast<hipStream_t>(hip_stream)));
}

rrm_status rrm_gated_ff_backward(const rrm_ff_desc* desc, const void* x, const void* wg, const void* wu, const void* g,
                                 const void* u, const void* dh, void* dx, void* dwg, void* dwu, void* workspace,
                                 size_t workspace_bytes, void* hip_stream) {
    if (rrm_status st = check(desc)) return st;
    const rrm_ff_desc& d = *desc;
    if ((dwg == nullptr) != (dwu == nullptr)) return record_failure(RRM_ERR_NULL, "dwg and dwu are made together");
    if (!dwg && (!dx || d.m == 0)) return RRM_OK;
    if (d.m > 0 && (!g || !u || !dh || (dwg && !x) || (dx && (!wg || !wu))))
        return record_failure(RRM_ERR_NULL, "x / wg / wu / g / u / dh is NULL");
    if (!reachable(1, 0, d.m, d.x_row) || !reachable(1, 0, d.f, d.wg_row) || !reachable(1, 0, d.f, d.wu_row) ||
        !reachable(1, 0, d.m, d.h_row) || !reachable(1, 0, d.m, d.gu_row) || !reachable(1, 0, d.m, d.dx_row) ||
        !reachable(1, 0, d.f, d.dwg_row) || !reachable(1, 0, d.f, d.dwu_row))
        return record_failure(RRM_ERR_SHAPE, "feed-forward: strides out of range");
    if ((dx && !apart(1, 0, d.m, d.dx_row, d.k)) || (dwg && (!apart(1, 0, d.f, d.dwg_row, d.k) || !apart(1, 0, d.f, d.dwu_row, d.k))))
        return record_failure(RRM_ERR_SHAPE, "feed-forward: two elements of an output lie at one place");
    const size_t e = d.unaligned ? 2 : 16;
    if (misaligned(x, e) || misaligned(wg, e) || misaligned(wu, e) || misaligned(g, 2) || misaligned(u, 2) || misaligned(dh, 2) ||
        misaligned(dx, 2) || misaligned(dwg, 2) || misaligned(dwu, 2))
        return record_failure(RRM_ERR_ALIGN, "feed-forward: a pointer is not aligned (to 16 bytes, to its element: see rrm_ff_desc)");
    if (rrm_status st = check_workspace(workspace, workspace_bytes, ff_scratch(d, true))) return st;
    return finish(launch_gated_ff_backward(d, x, wg, wu, g, u, dh, dx, dwg, dwu, workspace, static_cast<hipStream_t>(hip_stream)));
}

rrm_status rrm_aux_norm_layout(const rrm_norm_desc* desc, int backward, int layout[2]) {
    if (rrm_status st = check(desc)) return st;
    if (!layout) return record_failure(RRM_ERR_NULL, "layout is NULL");
    if (desc->n == 0 || desc->positions == 0) return record_failure(RRM_ERR_SHAPE, "group norm: nothing to do");
    norm_layout(*desc, backward != 0, layout);
    return RRM_OK;
}

rrm_status rrm_aux_scan_layout(const rrm_scan_desc* desc, int backward, int layout[2]) {
    if (rrm_status st = check(desc)) return st;
    if (!layout) return record_failure(RRM_ERR_NULL, "layout is NULL");
    if (desc->n == 0 || desc->c == 0) return record_failure(RRM_ERR_SHAPE, "gated scan: nothing to do");
    scan_layout(*desc, backward != 0, layout);
    return RRM_OK;
}

rrm_status rrm_aux_ff_layout(const rrm_ff_desc* desc, int asked, int layout[5]) {
    if (rrm_status st = check(desc)) return st;
    if (!layout) return record_failure(RRM_ERR_NULL, "layout is NULL");
    if (asked < 0 || asked > 3) return record_failure(RRM_ERR_OPTION, "feed-forward: asked is 0, or 1 (dX) + 2 (dW)");
    if (desc->m == 0) return record_failure(RRM_ERR_SHAPE, "feed-forward: nothing to do");
    ff_layout(*desc, asked, layout);
    return RRM_OK;
}

#pragma GCC visibility pop
}  // extern "C"
