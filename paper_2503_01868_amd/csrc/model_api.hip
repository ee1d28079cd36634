// C ABI of the operators around the mixers: argument validation (before any HIP call) and kernel selection.
#include "hy_checks.hpp"
#include "hy_common.hpp"
#include "hy_launch.hpp"

using namespace hy;

namespace {

constexpr int64_t kMostElements = INT64_C(1) << 60;  // of one tensor, gaps between its rows included

bool known(int32_t dtype) { return dtype == HY_F32 || dtype == HY_BF16; }

int64_t size_of(int32_t dtype) { return dtype == HY_F32 ? 4 : 2; }

// a * b * c <= kMostElements, for values that are not negative
bool fits(int64_t a, int64_t b, int64_t c) {
    return a == 0 || b == 0 || c == 0 || (a <= kMostElements / b && a * b <= kMostElements / c);
}

hy_status check_glr(int64_t B, int64_t L, int64_t D, int32_t group, int32_t dtype) {
    if (B < 0 || L < 0 || D < 0 || group < 1 || D % group != 0 || !fits(B, L + 1, D)) return HY_ERR_SHAPE;
    return known(dtype) ? HY_OK : HY_ERR_DTYPE;
}

GlrShape glr_shape(int64_t B, int64_t L, int64_t D, int32_t group, int32_t dtype) {
    GlrShape s{B, L, D, group, static_cast<hy_dtype>(dtype), {}, {}};
    for (int i = 0; i < 5; ++i) {
        s.rstride[i] = i == kGlrG ? D / group : D;
        s.bstride[i] = s.rstride[i] * L;
    }
    return s;
}

hy_status take_strides(GlrShape& s, const int64_t* strides, const int* which, int n) {
    if (!strides) return HY_OK;
    for (int i = 0; i < n; ++i) {
        const int64_t b = strides[2 * i], r = strides[2 * i + 1];
        if (b < 0 || r < 0) return HY_ERR_SHAPE;
        if (!fits(s.B > 1 ? s.B - 1 : 0, b, 1) || !fits(s.L > 1 ? s.L - 1 : 0, r, 1)) return HY_ERR_SHAPE;
        s.bstride[which[i]] = s.B > 1 ? b : 0;
        s.rstride[which[i]] = s.L > 1 ? r : 0;
    }
    return HY_OK;
}

Range glr_range(const GlrShape& s, const void* p, int i) {
    if (empty(s.B, s.L, s.D)) return Range{p, 0};
    const int64_t row = i == kGlrG ? s.D / s.group : s.D;
    return Range{p, ((s.B - 1) * s.bstride[i] + (s.L - 1) * s.rstride[i] + row) * size_of(s.dtype)};
}

hy_status all_aligned(const Range* r, int n) {
    for (int i = 0; i < n; ++i)
        if (!aligned16(r[i].p)) return HY_ERR_ALIGN;
    return HY_OK;
}

// Inputs may be views that begin at any element; from odd ones a lane takes one channel at a time.
hy_status take_starts(GlrShape& s, const Range* r, int n, int gate) {
    const uintptr_t e = (uintptr_t)size_of(s.dtype);
    for (int i = 0; i < n; ++i) {
        const uintptr_t at = reinterpret_cast<uintptr_t>(r[i].p);
        if (at % e != 0) return HY_ERR_ALIGN;
        if (at % (2 * e) != 0 && (i != gate || s.group == 1)) s.odd_start = true;
    }
    return HY_OK;
}

int64_t marks_bytes(const GlrShape& s) { return s.B * ((s.L + kGlrRows - 1) / kGlrRows) * s.D * 4; }

}  // namespace

extern "C" {

int64_t hyena_glr_fwd_workspace_bytes(int64_t B, int64_t L, int64_t D, int32_t group, int32_t dtype) {
    if (check_glr(B, L, D, group, dtype) != HY_OK) return -1;
    return empty(B, L, D) ? 0 : glr_fwd_workspace_bytes(glr_shape(B, L, D, group, dtype));
}

int64_t hyena_glr_bwd_workspace_bytes(int64_t B, int64_t L, int64_t D, int32_t group, int32_t dtype, int32_t with_marks) {
    if (check_glr(B, L, D, group, dtype) != HY_OK) return -1;
    return empty(B, L, D) ? 0 : glr_bwd_workspace_bytes(glr_shape(B, L, D, group, dtype), with_marks != 0);
}

hy_status hyena_glr_fwd(const void* q, const void* k, const void* v, const void* g, const float* state_in, void* y,
                        float* state_out, float* marks, const int64_t* strides, void* workspace, int64_t workspace_bytes,
                        int64_t B, int64_t L, int64_t D, int32_t group, int32_t dtype, void* hip_stream) {
    hy_status rc = check_glr(B, L, D, group, dtype);
    if (rc != HY_OK) return rc;
    if (!empty(B, L, D) && (!q || !k || !v || !g || !y)) return HY_ERR_NULL;
    if (workspace_bytes < 0) return HY_ERR_SHAPE;
    GlrShape s = glr_shape(B, L, D, group, dtype);
    const int which[4] = {kGlrQ, kGlrK, kGlrV, kGlrG};
    rc = take_strides(s, strides, which, 4);
    if (rc != HY_OK) return rc;
    const int64_t sb = B * D * 4;
    const Range rd[5] = {glr_range(s, q, kGlrQ), glr_range(s, k, kGlrK), glr_range(s, v, kGlrV), glr_range(s, g, kGlrG),
                         {state_in, state_in ? sb : 0}};
    const Range wr[3] = {{y, B * L * D * size_of(dtype)}, {state_out, state_out ? sb : 0}, {marks, marks ? marks_bytes(s) : 0}};
    rc = take_starts(s, rd, 4, 3);
    if (rc == HY_OK) rc = all_aligned(rd + 4, 1);
    if (rc == HY_OK) rc = all_aligned(wr, 3);
    if (rc == HY_OK) rc = check_disjoint(rd, 5, wr, 3);
    if (rc != HY_OK) return rc;
    if (B == 0 || D == 0 || (L == 0 && !state_out)) return HY_OK;
    const Range others[8] = {rd[0], rd[1], rd[2], rd[3], rd[4], wr[0], wr[1], wr[2]};
    rc = check_workspace(workspace, workspace_bytes, L > 0 ? glr_fwd_workspace_bytes(s) : 0, others, 8);
    if (rc != HY_OK) return rc;
    GlrPtrs p;
    p.q = q, p.k = k, p.v = v, p.g = g, p.state_in = state_in;
    p.y = y, p.state_out = state_out, p.marks_out = marks;
    return launch_glr_fwd(p, s, workspace, static_cast<hipStream_t>(hip_stream));
}

hy_status hyena_glr_bwd(const void* dy, const void* q, const void* k, const void* v, const void* g, const float* marks,
                        const float* state_in, const float* dstate_out, void* dq, void* dk, void* dv, void* dg,
                        float* dstate_in, const int64_t* strides, void* workspace, int64_t workspace_bytes, int64_t B, int64_t L,
                        int64_t D, int32_t group, int32_t dtype, void* hip_stream) {
    hy_status rc = check_glr(B, L, D, group, dtype);
    if (rc != HY_OK) return rc;
    if (!empty(B, L, D) && (!dy || !q || !k || !v || !g || !dq || !dk || !dv || !dg)) return HY_ERR_NULL;
    if (workspace_bytes < 0) return HY_ERR_SHAPE;
    GlrShape s = glr_shape(B, L, D, group, dtype);
    const int which[5] = {kGlrDy, kGlrQ, kGlrK, kGlrV, kGlrG};
    rc = take_strides(s, strides, which, 5);
    if (rc != HY_OK) return rc;
    const int64_t sb = B * D * 4, bytes = B * L * D * size_of(dtype);
    const Range rd[8] = {glr_range(s, dy, kGlrDy), glr_range(s, q, kGlrQ), glr_range(s, k, kGlrK), glr_range(s, v, kGlrV),
                         glr_range(s, g, kGlrG), {marks, marks ? marks_bytes(s) : 0}, {state_in, state_in ? sb : 0},
                         {dstate_out, dstate_out ? sb : 0}};
    const Range wr[5] = {{dq, bytes}, {dk, bytes}, {dv, bytes}, {dg, bytes / group}, {dstate_in, dstate_in ? sb : 0}};
    rc = take_starts(s, rd, 5, 4);
    if (rc == HY_OK) rc = all_aligned(rd + 5, 3);
    if (rc == HY_OK) rc = all_aligned(wr, 5);
    if (rc == HY_OK) rc = check_disjoint(rd, 8, wr, 5);
    if (rc != HY_OK) return rc;
    if (B == 0 || D == 0 || (L == 0 && !dstate_in)) return HY_OK;
    Range others[13];
    for (int i = 0; i < 8; ++i) others[i] = rd[i];
    for (int i = 0; i < 5; ++i) others[8 + i] = wr[i];
    rc = check_workspace(workspace, workspace_bytes, L > 0 ? glr_bwd_workspace_bytes(s, marks != nullptr) : 0, others, 13);
    if (rc != HY_OK) return rc;
    GlrPtrs p;
    p.dy = dy, p.q = q, p.k = k, p.v = v, p.g = g, p.marks = marks, p.state_in = state_in, p.dstate_out = dstate_out;
    p.dq = dq, p.dk = dk, p.dv = dv, p.dg = dg, p.dstate_in = dstate_in;
    return launch_glr_bwd(p, s, workspace, static_cast<hipStream_t>(hip_stream));
}

hy_status hyena_glr_step(const void* q, const void* k, const void* v, const void* g, float* state, void* y, int64_t B, int64_t D,
                         int32_t group, int32_t dtype, void* hip_stream) {
    hy_status rc = check_glr(B, 1, D, group, dtype);
    if (rc != HY_OK) return rc;
    if (!empty(B, 1, D) && (!q || !k || !v || !g || !state || !y)) return HY_ERR_NULL;
    const int64_t bytes = B * D * size_of(dtype);
    const Range rd[4] = {{q, bytes}, {k, bytes}, {v, bytes}, {g, bytes / group}};
    const Range wr[2] = {{y, bytes}, {state, B * D * 4}};
    GlrShape s = glr_shape(B, 1, D, group, dtype);
    rc = take_starts(s, rd, 4, 3);
    if (rc == HY_OK) rc = all_aligned(wr, 2);
    if (rc == HY_OK) rc = check_disjoint(rd, 4, wr, 2);
    if (rc != HY_OK || B == 0 || D == 0) return rc;
    GlrPtrs p;
    p.q = q, p.k = k, p.v = v, p.g = g, p.y = y, p.state_out = state;
    return launch_glr_step(p, s, static_cast<hipStream_t>(hip_stream));
}

}  // extern "C"
