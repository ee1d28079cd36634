// C ABI of linear attention, the RMS norm and the choice of tokens: argument validation (before any HIP call).
#include <algorithm>

#include "hy_common.hpp"
#include "hy_launch.hpp"
#include "hy_model_checks.hpp"

using namespace hy;

namespace {

// ---- linear attention

hy_status check_la(int64_t B, int64_t L, int64_t H, int32_t group, int64_t dk, int64_t dv, int32_t dtype) {
    if (B < 0 || L < 0 || H < 0 || dk < 1 || dv < 1 || group < 1 || H % group != 0 || L > kMostElements) return HY_ERR_SHAPE;
    // (also of what is empty: strides are computed all the same)
    const int64_t b = std::max<int64_t>(B, 1), h = std::max<int64_t>(H, 1), d = std::max(dk, dv);
    if (!fits(b, h, 1) || !fits(L + 1, d, 1) || !fits(b * h, L + 1, d) || !fits(dk, dv, 1) || !fits(b * h, dk, dv)) return HY_ERR_SHAPE;
    return known(dtype) ? HY_OK : HY_ERR_DTYPE;
}

LaShape la_shape(int64_t B, int64_t L, int64_t H, int32_t group, int64_t dk, int64_t dv, double scale, int32_t dtype) {
    LaShape s{B, L, H, group, dk, dv, scale, static_cast<hy_dtype>(dtype), {}};
    for (int i = 0; i < 5; ++i) {
        const int64_t heads = i == kLaQ || i == kLaK ? H / group : H, d = i == kLaQ || i == kLaK ? dk : i == kLaG ? 1 : dv;
        s.stride[i][2] = d, s.stride[i][1] = heads * d, s.stride[i][0] = heads * d * L;
    }
    return s;
}

int64_t heads_of(const LaShape& s, int which) { return which == kLaQ || which == kLaK ? s.H / s.group : s.H; }
int64_t width_of(const LaShape& s, int which) { return which == kLaQ || which == kLaK ? s.dk : which == kLaG ? 1 : s.dv; }

hy_status take_strides(LaShape& s, const int64_t* st, const int* which, int n) {
    if (!st) return HY_OK;
    for (int i = 0; i < n; ++i) {
        const int x = which[i];
        const int64_t many[3] = {s.B, s.L, heads_of(s, x)};
        for (int j = 0; j < (x == kLaG ? 2 : 3); ++j) {
            const int64_t d = *st++;
            if (d < 0 || !fits(many[j] > 1 ? many[j] - 1 : 0, d, 1)) return HY_ERR_SHAPE;
            s.stride[x][j] = many[j] > 1 ? d : 0;
        }
    }
    return HY_OK;
}

Range la_range(const LaShape& s, const void* p, int which) {
    if (s.B == 0 || s.L == 0 || s.H == 0) return Range{p, 0};
    const int64_t* st = s.stride[which];
    const int64_t last = (s.B - 1) * st[0] + (s.L - 1) * st[1] + (heads_of(s, which) - 1) * st[2];
    return Range{p, (last + width_of(s, which)) * size_of(s.dtype)};
}

hy_status on_elements(const Range* r, int n, int64_t bytes) {
    for (int i = 0; i < n; ++i)
        if (!on_element(r[i].p, bytes)) return HY_ERR_ALIGN;
    return HY_OK;
}

// ---- norm

hy_status check_norm(int64_t N, int64_t D, int32_t dtype) {
    if (N < 0 || D < 1 || !fits(std::max<int64_t>(N, 1), D, 1)) return HY_ERR_SHAPE;
    if (!known(dtype)) return HY_ERR_DTYPE;
    return D > INT32_MAX ? HY_ERR_UNSUPPORTED : HY_OK;
}

Range rows_range(const void* p, int64_t N, int64_t D, int64_t stride, int64_t bytes) {
    return Range{p, p && N > 0 ? ((N - 1) * stride + D) * bytes : 0};
}

}  // namespace

extern "C" {

int64_t hyena_la_marks_bytes(int64_t B, int64_t L, int64_t H, int32_t group, int64_t dk, int64_t dv, int32_t dtype) {
    if (check_la(B, L, H, group, dk, dv, dtype) != HY_OK) return -1;
    const LaShape s = la_shape(B, L, H, group, dk, dv, 1.0, dtype);
    return !la_served(s) ? -1 : empty(B, L, H) ? 0 : la_marks_bytes(s);
}

int64_t hyena_la_fwd_workspace_bytes(int64_t B, int64_t L, int64_t H, int32_t group, int64_t dk, int64_t dv, int32_t dtype) {
    if (check_la(B, L, H, group, dk, dv, dtype) != HY_OK) return -1;
    const LaShape s = la_shape(B, L, H, group, dk, dv, 1.0, dtype);
    return !la_served(s) ? -1 : empty(B, L, H) ? 0 : la_fwd_workspace_bytes(s);
}

int64_t hyena_la_bwd_workspace_bytes(int64_t B, int64_t L, int64_t H, int32_t group, int64_t dk, int64_t dv, int32_t dtype,
                                     int32_t with_marks) {
    if (check_la(B, L, H, group, dk, dv, dtype) != HY_OK) return -1;
    const LaShape s = la_shape(B, L, H, group, dk, dv, 1.0, dtype);
    return !la_served(s) ? -1 : empty(B, L, H) ? 0 : la_bwd_workspace_bytes(s, with_marks != 0);
}

hy_status hyena_la_fwd(const void* q, const void* k, const void* v, const void* g, const float* state_in, void* y, float* state_out,
                       void* marks, const int64_t* strides, void* workspace, int64_t workspace_bytes, int64_t B, int64_t L, int64_t H,
                       int32_t group, int64_t dk, int64_t dv, double scale, int32_t dtype, void* hip_stream) {
    hy_status rc = check_la(B, L, H, group, dk, dv, dtype);
    if (rc != HY_OK) return rc;
    if (!empty(B, L, H) && (!q || !k || !v || !g || !y)) return HY_ERR_NULL;
    if (workspace_bytes < 0) return HY_ERR_SHAPE;
    LaShape s = la_shape(B, L, H, group, dk, dv, scale, dtype);
    const int which[4] = {kLaQ, kLaK, kLaV, kLaG};
    rc = take_strides(s, strides, which, 4);
    if (rc != HY_OK) return rc;
    if (!la_served(s)) return HY_ERR_UNSUPPORTED;
    const int64_t sb = B * H * dk * dv * 4;
    const bool none = empty(B, L, H);
    const Range rd[5] = {la_range(s, q, kLaQ), la_range(s, k, kLaK), la_range(s, v, kLaV), la_range(s, g, kLaG),
                         {state_in, state_in ? sb : 0}};
    const Range wr[3] = {{y, B * L * H * dv * size_of(dtype)}, {state_out, state_out ? sb : 0}, {marks, marks && !none ? la_marks_bytes(s) : 0}};
    rc = on_elements(rd, 4, size_of(dtype));
    if (rc == HY_OK) rc = all_aligned(rd + 4, 1);
    if (rc == HY_OK) rc = all_aligned(wr, 3);
    if (rc == HY_OK) rc = check_disjoint(rd, 5, wr, 3);
    if (rc != HY_OK) return rc;
    if (B == 0 || H == 0 || (L == 0 && !state_out)) return HY_OK;
    const Range others[8] = {rd[0], rd[1], rd[2], rd[3], rd[4], wr[0], wr[1], wr[2]};
    rc = check_workspace(workspace, workspace_bytes, L > 0 ? la_fwd_workspace_bytes(s) : 0, others, 8);
    if (rc != HY_OK) return rc;
    LaPtrs p;
    p.q = q, p.k = k, p.v = v, p.g = g, p.state_in = state_in, p.y = y, p.state_out = state_out, p.marks = marks;
    return launch_la_fwd(p, s, workspace, static_cast<hipStream_t>(hip_stream));
}

hy_status hyena_la_bwd(const void* dy, const void* q, const void* k, const void* v, const void* g, const void* marks,
                       const float* state_in, const float* dstate_out, void* dq, void* dk, void* dv, void* dg, float* dstate_in,
                       const int64_t* strides, void* workspace, int64_t workspace_bytes, int64_t B, int64_t L, int64_t H, int32_t group,
                       int64_t d_k, int64_t d_v, double scale, int32_t dtype, void* hip_stream) {
    hy_status rc = check_la(B, L, H, group, d_k, d_v, dtype);
    if (rc != HY_OK) return rc;
    if (!empty(B, L, H) && (!dy || !q || !k || !v || !g || !dq || !dk || !dv || !dg)) return HY_ERR_NULL;
    if (workspace_bytes < 0) return HY_ERR_SHAPE;
    LaShape s = la_shape(B, L, H, group, d_k, d_v, scale, dtype);
    const int which[5] = {kLaDy, kLaQ, kLaK, kLaV, kLaG};
    rc = take_strides(s, strides, which, 5);
    if (rc != HY_OK) return rc;
    if (!la_served(s)) return HY_ERR_UNSUPPORTED;
    const bool none = empty(B, L, H);
    const int64_t sb = B * H * d_k * d_v * 4, e = size_of(dtype), rows = B * L * H;
    const Range rd[8] = {la_range(s, dy, kLaDy), la_range(s, q, kLaQ), la_range(s, k, kLaK), la_range(s, v, kLaV), la_range(s, g, kLaG),
                         {marks, marks && !none ? la_marks_bytes(s) : 0}, {state_in, state_in ? sb : 0}, {dstate_out, dstate_out ? sb : 0}};
    const Range wr[5] = {{dq, rows / group * d_k * e}, {dk, rows / group * d_k * e}, {dv, rows * d_v * e}, {dg, rows * e},
                         {dstate_in, dstate_in ? sb : 0}};
    rc = on_elements(rd, 5, e);
    if (rc == HY_OK) rc = all_aligned(rd + 5, 3);
    if (rc == HY_OK) rc = all_aligned(wr, 5);
    if (rc == HY_OK) rc = check_disjoint(rd, 8, wr, 5);
    if (rc != HY_OK) return rc;
    if (B == 0 || H == 0 || (L == 0 && !dstate_in)) return HY_OK;
    Range others[13];
    for (int i = 0; i < 8; ++i) others[i] = rd[i];
    for (int i = 0; i < 5; ++i) others[8 + i] = wr[i];
    rc = check_workspace(workspace, workspace_bytes, L > 0 ? la_bwd_workspace_bytes(s, marks != nullptr) : 0, others, 13);
    if (rc != HY_OK) return rc;
    LaPtrs p;
    p.dy = dy, p.q = q, p.k = k, p.v = v, p.g = g, p.marks_in = marks, p.state_in = state_in, p.dstate_out = dstate_out;
    p.dq = dq, p.dk = dk, p.dv = dv, p.dg = dg, p.dstate_in = dstate_in;
    return launch_la_bwd(p, s, workspace, static_cast<hipStream_t>(hip_stream));
}

hy_status hyena_la_step(const void* q, const void* k, const void* v, const void* g, float* state, void* y, int64_t B, int64_t H,
                        int32_t group, int64_t dk, int64_t dv, double scale, int32_t dtype, void* hip_stream) {
    hy_status rc = check_la(B, 1, H, group, dk, dv, dtype);
    if (rc != HY_OK) return rc;
    const bool none = B == 0 || H == 0;
    if (!none && (!q || !k || !v || !g || !state || !y)) return HY_ERR_NULL;
    const int64_t slices = (dv + 31) / 32, most = INT64_C(1) << 23;
    if (dk > 65536 || (!none && (B >= most || H >= most || slices >= most || B * H >= most || B * H * slices >= most))) return HY_ERR_UNSUPPORTED;
    const LaShape s = la_shape(B, 1, H, group, dk, dv, scale, dtype);
    const int64_t e = size_of(dtype);
    const Range rd[4] = {{q, B * H / group * dk * e}, {k, B * H / group * dk * e}, {v, B * H * dv * e}, {g, B * H * e}};
    const Range wr[2] = {{y, B * H * dv * e}, {state, B * H * dk * dv * 4}};
    rc = on_elements(rd, 4, e);
    if (rc == HY_OK) rc = all_aligned(wr, 2);
    if (rc == HY_OK) rc = check_disjoint(rd, 4, wr, 2);
    if (rc != HY_OK || none) return rc;
    LaPtrs p;
    p.q = q, p.k = k, p.v = v, p.g = g, p.y = y, p.state_out = state;
    return launch_la_step(p, s, static_cast<hipStream_t>(hip_stream));
}

hy_status hyena_rmsnorm_fwd(const void* x, const void* residual, const void* w, void* y, float* y_scale, void* h, float* rstd, int64_t N,
                            int64_t D, int64_t x_stride, int64_t r_stride, double eps, int32_t dtype, void* hip_stream) {
    hy_status rc = check_norm(N, D, dtype);
    if (rc != HY_OK) return rc;
    if (x_stride < 0 || !(eps >= 0) || (residual && r_stride < 0) || (h && !residual)) return HY_ERR_SHAPE;
    if (!residual || N <= 1) r_stride = 0;
    if (N <= 1) x_stride = 0;
    if (!fits(N, x_stride, 1) || !fits(N, r_stride, 1)) return HY_ERR_SHAPE;
    if (N == 0) return HY_OK;
    if (!x || !y) return HY_ERR_NULL;
    const int64_t e = size_of(dtype);
    const Range rd[3] = {rows_range(x, N, D, x_stride, e), rows_range(residual, N, D, r_stride, e), {w, w ? D * e : 0}};
    const Range wr[4] = {{y, N * D * (y_scale ? 1 : e)}, {y_scale, y_scale ? N * 4 : 0}, {rstd, rstd ? N * 4 : 0}, {h, h ? N * D * e : 0}};
    for (const Range& r : rd)
        if (!on_element(r.p, e)) return HY_ERR_ALIGN;
    if (!on_element(y, y_scale ? 1 : e) || !on_element(y_scale, 4) || !on_element(rstd, 4) || !on_element(h, e)) return HY_ERR_ALIGN;
    rc = check_disjoint(rd, 3, wr, 3);
    if (rc != HY_OK) return rc;
    if (h) {  // in place on dense rows of x or of the residual, apart from everything else
        Range others[5] = {rd[0], rd[1], rd[2], wr[0], wr[1]};
        const int64_t st[2] = {x_stride, r_stride};
        for (int i = 0; i < 2; ++i)
            if (others[i].p == h && (N == 1 || st[i] == D)) others[i].bytes = 0;
        rc = check_disjoint(others, 5, wr + 3, 1);
        if (rc == HY_OK) rc = check_disjoint(wr + 2, 1, wr + 3, 1);
        if (rc != HY_OK) return rc;
    }
    NormPtrs p;
    p.x = x, p.residual = residual, p.w = w, p.y = y, p.y_scale = y_scale, p.h = h, p.rstd = rstd;
    return launch_norm_fwd(p, NormShape{N, D, x_stride, r_stride, eps, dtype}, static_cast<hipStream_t>(hip_stream));
}

int64_t hyena_rmsnorm_bwd_workspace_bytes(int64_t N, int64_t D, int32_t dtype) {
    return check_norm(N, D, dtype) != HY_OK ? -1 : norm_bwd_workspace_bytes(N, D);
}

hy_status hyena_rmsnorm_bwd(const void* dy, const void* h, const float* rstd, const void* w, const void* dh, void* dx, void* dw,
                            void* workspace, int64_t workspace_bytes, int64_t N, int64_t D, int32_t dtype, void* hip_stream) {
    hy_status rc = check_norm(N, D, dtype);
    if (rc != HY_OK) return rc;
    if (workspace_bytes < 0 || (dw && !w)) return HY_ERR_SHAPE;
    if (N > 0 && (!dy || !h || !rstd || !dx)) return HY_ERR_NULL;
    const int64_t e = size_of(dtype), bytes = N * D * e;
    const Range rd[5] = {{dy, bytes}, {h, bytes}, {rstd, N * 4}, {w, w ? D * e : 0}, {dh, dh ? bytes : 0}};
    const Range wr[2] = {{dx, bytes}, {dw, dw ? D * e : 0}};
    if (!on_element(dy, e) || !on_element(h, e) || !on_element(rstd, 4) || !on_element(w, e) || !on_element(dh, e) || !on_element(dx, e) ||
        !on_element(dw, e))
        return HY_ERR_ALIGN;
    Range others[5] = {rd[0], rd[1], rd[2], rd[3], rd[4]};
    for (int i : {0, 4})
        if (others[i].p == dx) others[i].bytes = 0;
    rc = check_disjoint(others, 5, wr, 1);
    if (rc == HY_OK) rc = check_disjoint(rd, 5, wr + 1, 1);
    if (rc == HY_OK) rc = check_disjoint(wr, 1, wr + 1, 1);
    if (rc != HY_OK) return rc;
    if (dw && N > 0) {
        const Range all[7] = {rd[0], rd[1], rd[2], rd[3], rd[4], wr[0], wr[1]};
        rc = check_workspace(workspace, workspace_bytes, norm_bwd_workspace_bytes(N, D), all, 7);
        if (rc != HY_OK) return rc;
    }
    if (N == 0 && !dw) return HY_OK;
    NormPtrs p;
    p.dy = dy, p.h = const_cast<void*>(h), p.rstd = const_cast<float*>(rstd), p.w = w, p.dh = dh, p.dx = dx, p.dw = dw;
    return launch_norm_bwd(p, NormShape{N, D, 0, 0, 0.0, dtype}, workspace, static_cast<hipStream_t>(hip_stream));
}

hy_status hyena_sample(const void* logits, const float* u, const float* temperature, double temperature_all, const int32_t* top_k,
                       int32_t top_k_all, const float* top_p, double top_p_all, const float* min_p, double min_p_all, int64_t* token,
                       float* prob, int64_t N, int64_t V, int64_t stride, int32_t dtype, void* hip_stream) {
    if (N < 0 || V < 1 || stride < 0 || !fits(std::max<int64_t>(N, 1), V, 1)) return HY_ERR_SHAPE;
    if (N <= 1) stride = 0;
    if (!fits(N, stride, 1)) return HY_ERR_SHAPE;
    if (!known(dtype)) return HY_ERR_DTYPE;
    const int64_t most = INT64_C(1) << 22;
    if (N > most || V > most) return HY_ERR_UNSUPPORTED;
    if (N == 0) return HY_OK;
    if (!logits || !u || !token) return HY_ERR_NULL;
    const int64_t e = size_of(dtype);
    const Range rd[6] = {rows_range(logits, N, V, stride, e), {u, N * 4}, {temperature, temperature ? N * 4 : 0}, {top_k, top_k ? N * 4 : 0},
                         {top_p, top_p ? N * 4 : 0}, {min_p, min_p ? N * 4 : 0}};
    const Range wr[2] = {{token, N * 8}, {prob, prob ? N * 4 : 0}};
    if (!on_element(logits, e) || !on_element(token, 8) || !on_element(prob, 4)) return HY_ERR_ALIGN;
    hy_status rc = on_elements(rd + 1, 5, 4);
    if (rc == HY_OK) rc = check_disjoint(rd, 6, wr, 2);
    if (rc != HY_OK) return rc;
    return launch_sample(SamplePtrs{logits, u, temperature, top_p, min_p, top_k, token, prob},
                         SampleAll{temperature_all, top_p_all, min_p_all, top_k_all}, N, V, stride, dtype,
                         static_cast<hipStream_t>(hip_stream));
}

}  // extern "C"
